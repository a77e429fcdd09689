"""Norm and rotation: what a head's result depends on, its range, and the precision of the sums.

Bounds as in test_gpu_rope.  Of the norm alone (nothing turned): the sum of squares in float64, its
factor brought to float32 (half a step, 2^-24), its product with the entry and the gain's, half a step each:
  |out - ref| <= 3.01 2^-24 |y|
"""
import numpy as np
import pytest

from oracle import rope as oracle
from paper_2608_10362_amd import binding
from tests.gpu_util import f32, i32, log, torch_cuda
from tests.test_gpu_fp8_cache import _cache, _np, _shape
from tests.test_gpu_rope import EPS, _compare, _tol

pytestmark = pytest.mark.gpu


def _bad_heads(x, heads):
    """Heads of x [batch, n, heads, hd] that leave float32's range for squares, each in a way of its own."""
    for h, kind in zip(heads, range(5)):
        if kind < 3:
            x[:, :, h] *= (2.0 ** 110, 2.0 ** -130, 0.0)[kind]
        elif kind == 3:
            x[:, :, h, 1] = np.nan
        else:
            x[:, :, h, 2] = np.inf
    return x


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("eps", [0.0, EPS])
def test_a_heads_bits_are_its_own(hd, interleaved, eps):
    """A head's result is the same bits alone and among heads of zeros, NaN, infinities and far magnitudes."""
    torch = torch_cuda()
    rng = np.random.default_rng(hd)
    B, n, H = 2, 11, 40
    g = f32(1 + rng.normal(0, 0.2, hd))
    r = binding.Rope(hd, interleaved=interleaved, q_gain=g, k_gain=g, eps=eps)
    x = rng.normal(0, 1.3, (B, n, H, hd)).astype(np.float32)
    bad = [1, 6, 12, 21, 30]
    good = [h for h in range(H) if h not in bad]
    pos = i32(rng.integers(0, 5000, (B, n)))
    alone = torch.empty((B, n, len(good), hd), device="cuda")
    binding.specdec_rope_apply(r, f32(x[:, :, good]), None, alone, None, positions=pos)
    among = torch.empty((B, n, H, hd), device="cuda")
    log(f"a head's own bits hd={hd} interleaved={interleaved} eps={eps}")
    binding.specdec_rope_apply(r, f32(_bad_heads(x.copy(), bad)), None, among, None, positions=pos)
    assert torch.equal(among[:, :, good], alone)
    # keys into a cache: rows of one head beside bad rows of it
    kv = _cache(_shape(hd, H, H, 1), B, 128, 128)
    kv.set_state([3, 8], [[0, 1]] * B, [1] * B)
    k = x.copy()
    rows = [t for t in range(n) if t not in (2, 9)]
    k[:, 2], k[:, 9] = 0.0, np.nan
    out = torch.empty((B, n, H, hd), device="cuda")
    binding.specdec_rope_append(kv, 0, r, f32(x), f32(k), f32(x), out, positions=pos)
    want = torch.empty((B, n, H, hd), dtype=torch.bfloat16, device="cuda")
    binding.specdec_rope_apply(r, None, f32(x), None, want, positions=pos)
    for b, L in enumerate([3, 8]):
        got = kv.read_context(0, b, L, n)[0]
        assert torch.equal(got[rows], want[b][rows])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("eps", [0.0, 1e-29, EPS])
@pytest.mark.parametrize("x_exp,g_exp", [(-140, 0), (-130, 20), (40, 100), (-40, -100), (49, 70), (120, -60), (0, 120)])
def test_far_magnitudes_alone(x_exp, g_exp, eps, interleaved):
    """Entries and gains far from 1, in every head of the call: no step in between overflows or vanishes where
    the result does not."""
    torch = torch_cuda()
    rng = np.random.default_rng(x_exp + 1000)
    hd, n, H = 64, 3, 8
    eps = float(np.float32(eps))
    x = (rng.normal(0, 1, (1, n, H, hd)) * 2.0 ** x_exp).astype(np.float32)
    g = (rng.normal(1, 0.1, hd) * 2.0 ** g_exp).astype(np.float32)
    out = torch.empty((1, n, H, hd), device="cuda")
    log(f"far magnitudes 2^{x_exp}, gains 2^{g_exp}, eps {eps}")
    binding.specdec_rope_apply(binding.Rope(hd, interleaved=interleaved, q_gain=f32(g), eps=eps), f32(x), None, out, None,
                               offset=5)
    if abs(g_exp) <= 20 and x_exp < -126 and eps:  # (a normalised value that is not normal: its half step, times the gain)
        y = oracle.norm(x, g, eps)
        ref, tol = _tol(x, 5 + np.arange(n)[None], oracle.freqs(hd, 10000.0), interleaved, g, eps, "f32")
        assert (np.abs(_np(out) - ref) <= tol + 2.0 ** -147 * (1 + 2.0 ** g_exp)).all(), np.abs(_np(out) - ref).max()
        assert np.isfinite(y).all()
    else:
        _compare(out, x, 5 + np.arange(n)[None], oracle.freqs(hd, 10000.0), interleaved, g, eps, "f32")


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_the_norms_own_precision(hd):
    torch = torch_cuda()
    rng = np.random.default_rng(hd)
    x = rng.normal(0, 1.3, (1, 400, 64, hd)).astype(np.float32)
    g = (1 + rng.normal(0, 0.2, hd)).astype(np.float32)
    out = torch.empty(x.shape, device="cuda")
    binding.specdec_rope_apply(binding.Rope(hd, rotary_dim=0, q_gain=f32(g), eps=EPS), f32(x), None, out, None)
    y = oracle.norm(x, g, float(np.float32(EPS)))
    worst = (np.abs(_np(out) - y) / np.abs(y)).max() * 2.0 ** 24
    log(f"norm alone, hd={hd}: worst {worst:.3g} of 2^-24")
    assert worst <= 3.01
