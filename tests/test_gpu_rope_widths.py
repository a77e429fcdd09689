"""Rotary widths of any multiple of 16: halves that are no power of two lanes apart, alone and into a cache, against
the float64 oracle (the bounds of test_gpu_rope)."""
import numpy as np
import pytest

from oracle import rope as oracle
from paper_2608_10362_amd import binding
from tests.gpu_util import i32, torch_cuda
from tests.test_gpu_fp8_cache import _cache, _np, _shape
from tests.test_gpu_rope import EPS, _compare, _inputs, _t, _type

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd,rot", [(64, 48), (128, 48), (128, 80), (128, 96), (128, 112)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norms", ["qk", "", "k"])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16")])
def test_rotary_widths(hd, rot, interleaved, norms, dtype, out):
    torch = torch_cuda()
    rng = np.random.default_rng(rot)
    B, n, H, G, lens = 2, 13, 10, 5, [5, 64]
    q, k, v = _inputs(rng, B, n, H, G, hd, dtype, lead=1)
    gq, gk = (_t(1 + rng.normal(0, 0.2, hd), dtype) if s in norms else None for s in "qk")
    r = binding.Rope(hd, rotary_dim=rot, interleaved=interleaved, q_gain=gq, k_gain=gk, eps=EPS)
    freq = oracle.freqs(rot, 10000.0)
    pos = np.array(lens)[:, None] + np.arange(n) + 900
    q_out, k_out = (torch.full(x.shape, float("nan"), dtype=_type(out), device="cuda") for x in (q, k))
    binding.specdec_rope_apply(r, q, k, q_out, k_out, positions=i32(pos))
    gains = [None if g is None else _np(g) for g in (gq, gk)]
    _compare(q_out, _np(q), pos, freq, interleaved, gains[0], EPS, out)
    _compare(k_out, _np(k), pos, freq, interleaved, gains[1], EPS, out)
    kv = _cache(_shape(hd, H, G, 1), B, 128, 128)
    kv.set_state(lens, [[0, 1]] * B, [1] * B)
    again = torch.full(q.shape, float("nan"), dtype=_type(out), device="cuda")
    binding.specdec_rope_append(kv, 0, r, q, k, v, again, offset=900)
    assert torch.equal(again, q_out)
    keys = torch.empty(k.shape, dtype=torch.bfloat16, device="cuda")
    binding.specdec_rope_apply(r, None, k, None, keys, positions=i32(pos))
    for b, L in enumerate(lens):
        rows = kv.read_context(0, b, L, n)
        assert torch.equal(rows[0], keys[b]) and torch.equal(rows[1], v[b].to(torch.bfloat16))
