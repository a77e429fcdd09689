"""Calls of specdec_attention beside those of tests/test_gpu_fp8_cache.py."""
import numpy as np
import pytest

from oracle import fp8
from paper_2608_10362_amd import binding
from tests import fp8_parts
from tests.gpu_util import log
from tests.test_gpu_fp8_cache import _attend, _bf16, _cache, _check, _np, _shape

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("n", [1, 70])
@pytest.mark.parametrize("L,out", [(700, slice(0, 256)), (3000, slice(0, 1024)), (700, slice(690, 700)), (150, slice(64, 150))])
def test_scores_below_float32(hd, n, L, out):
    """Keys whose score is below float32's range have the weight 0, whichever wave or
    part has no others: -2^132 / sqrt(hd) for the rows `out`, whole blocks of codes or rows of the ring."""
    rng = np.random.default_rng(hd + n + L)
    G, H, window = 1, 2, 192
    kv = _cache(_shape(hd, H, G, 1), 1, (L + n + 63) // 64 * 64, window)
    k, v = rng.normal(0, 1.3, (L + n, G, hd)), rng.normal(0, 1.3, (L + n, G, hd))
    k[:, :, 0] = 0
    k[out] = 0
    k[out, :, 0] = -2.0 ** 118
    k, v = _np(_bf16(k)), _np(_bf16(v))
    kv.write_context(0, 0, 0, _bf16(k[:L]), _bf16(v[:L]))
    kv.set_state([L], [[0, 1]], [1])
    binding.specdec_kv_append(kv, 0, _bf16(k[None, L:]), _bf16(v[None, L:]))
    q = rng.normal(0, 1.5, (1, n, H, hd)).astype(np.float32)
    q[..., 0] = 2.0 ** 14
    log(f"scores below float32: hd={hd} n={n} L={L} rows {out.start}..{out.stop}")
    got = _attend(kv, q)
    k, v = fp8.stored(k, L // 64 * 64), fp8.stored(v, L // 64 * 64)
    # (without those rows, and without the dimension that is 0 in all others)
    keep = np.r_[0:out.start, out.stop:L + n]
    q[..., 0] = 0
    log(f"worst error {_check(got, q, [[k[keep], v[keep]]], [L - (out.stop - out.start)]):.3g}")


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("kind", ["scores", "probabilities"])
@pytest.mark.parametrize("L", [60, 128], ids=["ring", "codes"])
@pytest.mark.parametrize("n,H", [(1, 64), (70, 2)], ids=["one tile", "two tiles"])
def test_parts_of_queries_and_probabilities(hd, kind, L, n, H):
    """Queries and probabilities reach the products whole: the bound of tests/fp8_parts.py,
    which a part less would break (tests/test_fp8_attention_parts.py)."""
    q, k, v, s1, s2 = fp8_parts.inputs(kind, hd, H, n, L + n, seed=hd + n + L)
    kv = _cache(_shape(hd, H, 1, 1), 1, 256, 192)
    k, v = k[:, None], v[:, None]
    kv.write_context(0, 0, 0, _bf16(k[:L]), _bf16(v[:L]))
    kv.set_state([L], [[0, 1]], [1])
    binding.specdec_kv_append(kv, 0, _bf16(k[None, L:]), _bf16(v[None, L:]))
    for x, stored in zip(kv.read_context(0, 0, 0, L), (k, v)):  # (powers of two: exact in codes)
        np.testing.assert_array_equal(_np(x), stored[:L])
    got = _attend(kv, q[None])[0]
    ref, tol = fp8_parts.reference(s1, s2), fp8_parts.bound(s1, s2)
    err = np.abs(got - ref[..., None]).max(-1)
    log(f"parts {kind} hd={hd} L={L} n={n}: worst {err.max():.3g}, {(err / tol).max():.3g} of the bound")
    assert (err <= tol).all()
