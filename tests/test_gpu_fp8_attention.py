"""Calls of specdec_attention beside those of tests/test_gpu_fp8_cache.py."""
import numpy as np
import pytest

from oracle import fp8
from paper_2608_10362_amd import binding
from tests import fp8_parts
from tests.gpu_util import log, torch_cuda
from tests.test_gpu_fp8_cache import _attend, _bf16, _cache, _check, _fill, _np, _shape

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


def _bad_rows(kv, rng, L, n, G, hd, rows):
    """Appends n rows, some with a NaN or infinity: rows[r] = (kind, kv head) of row L + r."""
    k, v = (_np(_bf16(rng.normal(0, 1.3, (n, G, hd)))) for _ in range(2))
    kb, vb = k.copy(), v.copy()
    for r, (kind, g) in rows.items():
        if kind == "k":
            kb[r, g, 2] = np.nan
        else:
            vb[r, g, 5], vb[r, g, 6] = (np.nan, -np.inf) if kind == "nan" else (np.inf, -np.inf)
    binding.specdec_kv_append(kv, 0, _bf16(kb[None]), _bf16(vb[None]))
    return k, v


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("n,H,L", [(70, 4, 150), (100, 2, 407), (66, 8, 63), (129, 2, 0)])
def test_many_rows_and_rows_that_are_not_seen(hd, n, H, L):
    """More than 64 query rows a kv head (two tiles a wave): NaN and infinities in K and V
    rows of the ring, which wraps, affect the queries that see them and no others, in
    every sub-chunk; slots past the newest row hold NaN."""
    rng = np.random.default_rng(hd + n + L)
    G, group = 2, H // 2
    assert n * group > 64
    window = (63 + n + 63) // 64 * 64
    kv = _cache(_shape(hd, H, G, 1), 1, (L + n + 63) // 64 * 64 + 64, window)
    ck, cv = (_np(_bf16(rng.normal(0, 1.3, (L, G, hd)))) for _ in range(2))
    if L:
        kv.write_context(0, 0, 0, _bf16(ck), _bf16(cv))
    kv.set_state([L], [[0, 1]], [1])
    # kv head 0: values; kv head 1: a key
    first, last, key = n // 7, n - 2, n // 2
    rows = {first: ("inf", 0), n // 3: ("nan", 0), (2 * n) // 3: ("inf", 0), last: ("nan", 0), key: ("k", 1)}
    k, v = _bad_rows(kv, rng, L, n, G, hd, rows)
    log(f"rows not seen: hd={hd} n={n} L={L} ring of {window}, bad rows {sorted(rows)}")
    q = rng.normal(0, 1, (1, n, H, hd)).astype(np.float32)
    got = _attend(kv, q)
    sealed = L // 64 * 64
    keys = np.concatenate([fp8.stored(ck, sealed), k]) if L else k.astype(np.float64)
    values = np.concatenate([fp8.stored(cv, sealed), v]) if L else v.astype(np.float64)
    h0, h1 = slice(0, group), slice(group, H)
    one = lambda x, g: x[:, g:g + 1]  # noqa: E731
    # rows before the first bad value, all dims; every row, the dims without one
    _check(got[:, :, h0], q[:, :, h0], [[one(keys, 0), one(values, 0)]], [L], rows=range(first))
    assert not np.isfinite(got[0, first:, h0, 5]).any() and not np.isfinite(got[0, first:, h0, 6]).any()
    clean, cut = got[:, :, h0].copy(), one(values, 0).copy()
    clean[..., 5:7], cut[..., 5:7] = 0, 0
    _check(clean, q[:, :, h0], [[one(keys, 0), cut]], [L])
    _check(got[:, :, h1], q[:, :, h1], [[one(keys, 1), one(values, 1)]], [L], rows=range(key))
    assert np.isnan(got[0, key:, h1]).all()
    assert kv.read_state()["status"] == 0


@pytest.mark.parametrize("case", [
    (128, 7, 1, [333], 1), (64, 71, 1, [200], 1), (32, 128, 1, [700], 1), (64, 128, 1, [90, 4000], 2),
    (128, 142, 2, [130], 3), (32, 34, 17, [64, 0, 65], 7)], ids=lambda c: f"hd{c[0]}-{c[1]}:{c[2]}-n{c[4]}")
def test_odd_groups_and_the_largest(case):
    """Query heads per kv head of 3 to 128, the last length up to the capacity, the second of two layers."""
    hd, H, G, lens, n = case
    rng = np.random.default_rng(H + n)
    cap = (max(lens) + n + 63) // 64 * 64
    lens = [cap - n if x == max(lens) else x for x in lens]  # (the longest fills the cache)
    kv = _cache(_shape(hd, H, G, 2), len(lens), cap, 128)
    _fill(kv, rng, lens, n, G, hd, layer=0)
    kvs = _fill(kv, rng, lens, n, G, hd, layer=1)
    q = rng.normal(0, 1.5, (len(lens), n, H, hd)).astype(np.float32)
    log(f"groups {case}: worst error {_check(_attend(kv, q, 1), q, kvs, lens):.3g}")
    binding.specdec_kv_advance(kv, n)
    assert kv.read_state()["status"] == 0


def test_two_caches_on_two_streams():
    """Calls at once on two caches, with workspaces of their own, eager and captured."""
    torch = torch_cuda()
    rng = np.random.default_rng(3)
    hd, H, G, n = 64, 8, 1, 2
    lens = [[5000, 17], [333, 2048]]
    kvs = [_cache(_shape(hd, H, G, 1), 2, 5056, 128) for _ in lens]
    held = [_fill(kv, rng, L, n, G, hd) for kv, L in zip(kvs, lens)]
    q = [torch.from_numpy(rng.normal(0, 1.5, (2, n, H, hd)).astype(np.float32)).cuda() for _ in lens]
    out = [torch.empty_like(x) for x in q]
    ws = [binding.attention_workspace(kv, H, n) for kv in kvs]
    streams, graphs = [torch.cuda.Stream() for _ in lens], []
    torch.cuda.synchronize()
    for j in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[j]):
            binding.specdec_attention(kvs[j], 0, q[j], out[j], ws[j])
        graphs.append(g)
    for rep in range(4):
        for o in out:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        log(f"two caches at once, {rep}")
        for i in range(5):
            for j in range(2):
                if rep % 2:
                    binding.specdec_attention(kvs[j], 0, q[j], out[j], ws[j], stream=streams[j])
                else:
                    with torch.cuda.stream(streams[j]):
                        graphs[j].replay()
        torch.cuda.synchronize()
        for j in range(2):
            _check(out[j].cpu().numpy(), q[j].cpu().numpy(), held[j], lens[j])


def test_lengths_set_back_and_grown_again():
    """A length set back (drafted text thrown away) and grown by other rows: codes of blocks that are
    completed anew, the ring's of those that are not, for a ring that has wrapped."""
    rng = np.random.default_rng(9)
    hd, H, G, window, cap = 64, 4, 2, 192, 640
    kv = _cache(_shape(hd, H, G, 1), 1, cap, window)
    k, v = (rng.normal(0, 1.3, (cap, G, hd)) for _ in range(2))
    k, v = _np(_bf16(k)), _np(_bf16(v))
    L = 500
    kv.write_context(0, 0, 0, _bf16(k[:L]), _bf16(v[:L]))
    for back in (500, 449, 447, 400, 380):
        kv.set_state([back], [[0, 1]], [1])
        n = 5
        k2, v2 = (_np(_bf16(rng.normal(0, 1.3, (n, G, hd)))) for _ in range(2))
        binding.specdec_kv_append(kv, 0, _bf16(k2[None]), _bf16(v2[None]))
        k[back:back + n], v[back:back + n] = k2, v2
        q = rng.normal(0, 1.5, (1, n, H, hd)).astype(np.float32)
        sealed = back // 64 * 64
        log(f"set back to {back}")
        _check(_attend(kv, q), q, [[fp8.stored(k[:back + n], sealed), fp8.stored(v[:back + n], sealed)]], [back])
        binding.specdec_kv_advance(kv, n)
        now = (back + n) // 64 * 64
        for got, x in zip(kv.read_context(0, 0, 0, back + n), (k, v)):
            np.testing.assert_array_equal(_np(got), fp8.stored(x[:back + n], now))
