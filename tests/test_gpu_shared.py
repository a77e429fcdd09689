"""Attention over a shared prefix, against a plain computation in 64 bits.

Both caches' values are exact (tests/test_gpu_fp8_cache.py), so the reference is the softmax over the
prefix's and the row's own stored keys.  The bound, of float32 queries and results, is
that file's (the parts of queries and probabilities, float32 sums) with the join's
exponentials and sums:
  ds  = (2^-18 + (hd + 2) 2^-24) max_j sum_d |q_d k_jd| / sqrt(hd) + 2^-22 max|s|
  |o - ref| <= (2 ds + 2^-17 + 2^-21 + (keys + 128) 2^-24) max|v|
bfloat16: a probability may enter its product and the sum as one fp16 value, off by half a step of
it, 2^-11, and below 2^-25 of the largest by half of 2^-24 2^-11 (which is 1 / 2^36 of it):
sum (p + e) v / sum (p + e) - o = sum e (v - o) / sum (p + e), at most 2 2^-11 (1 + 2^-10) max|v|,
and keys 2^-35 max|v|; the result is rounded to bfloat16, half a step, 2^-8 of it.
"""
import numpy as np
import pytest

from oracle import fp8
from oracle import rope as rope_oracle
from paper_2608_10362_amd import binding
from tests.gpu_util import f32, log, torch_cuda
from tests.test_gpu_fp8_cache import _bf16, _cache, _fill, _np, _rows, _shape

pytestmark = pytest.mark.gpu


def _prefix(rng, hd, G, P, batch=2, at=1, n_layers=2, cap=None, window=128, layer=0, spread=False):
    """A cache whose sequence `at` holds P rows in `layer`, and what they are."""
    kv = _cache(_shape(hd, 2 * G, G, n_layers), batch, max(64, cap or (P + 63) // 64 * 64), window)
    k, v = _rows(rng, P, G, hd, spread), _rows(rng, P, G, hd, spread)
    if P:
        kv.write_context(layer, at, 0, _bf16(k), _bf16(v))
    lens = [0] * batch
    lens[at] = P
    kv.set_state(lens, [[0, 1]] * batch, [1] * batch)
    return kv, fp8.stored(k, P // 64 * 64), fp8.stored(v, P // 64 * 64)


def _queries(rng, shape, dtype, sigma=1.5):
    torch = torch_cuda()
    q = f32(rng.normal(0, sigma, shape))
    return q.to(torch.bfloat16) if dtype == "bf16" else q


def _attend(prefix, kv, q, layer=0, at=1, ws=None, **more):
    torch = torch_cuda()
    out = torch.full_like(q, float("nan"))
    binding.specdec_attention_shared(prefix, kv, layer, q, out, workspace=ws, prefix_b=at, **more)
    return out


def _reference(q, pk, pv, kvs, lens):
    """ref [B, n, H, hd] and the bound [B, n, H, 1] of float32 results."""
    torch = torch_cuda()
    B, n, H, hd = q.shape
    d = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.float64)).cuda()  # noqa: E731
    ref, tol = torch.empty((B, n, H, hd), dtype=torch.float64, device="cuda"), None
    tol = torch.empty((B, n, H, 1), dtype=torch.float64, device="cuda")
    for b in range(B):
        k, v = (torch.cat([d(x), d(y)]).transpose(0, 1).contiguous() for x, y in zip((pk, pv), kvs[b]))  # [G, m, hd]
        G, m, P = k.shape[0], k.shape[1], len(pk)
        qb = q[b].double().reshape(n, G, H // G, hd).permute(1, 2, 0, 3).reshape(G, -1, hd)
        late = torch.arange(m, device="cuda")[None] > P + lens[b] + torch.arange(n, device="cuda")[:, None]
        late = late.repeat(H // G, 1)[None].expand(G, -1, -1)
        kt = k.transpose(1, 2).contiguous()
        s = torch.matmul(qb, kt) / np.sqrt(hd)
        mag = (torch.matmul(qb.abs(), kt.abs()) / np.sqrt(hd)).masked_fill(late, 0).amax(-1)
        ds = (2.0 ** -18 + (hd + 2) * 2.0 ** -24) * mag + 2.0 ** -22 * s.abs().masked_fill(late, 0).amax(-1)
        o = torch.matmul(torch.softmax(s.masked_fill(late, -float("inf")), -1), v)
        big = v.abs().amax((1, 2))[:, None]
        t = (2 * ds + 2.0 ** -17 + 2.0 ** -21 + (m + 128) * 2.0 ** -24) * big
        back = lambda x: x.reshape(G, H // G, n, -1).permute(2, 0, 1, 3).reshape(n, H, -1)  # noqa: E731
        ref[b], tol[b] = back(o), back(t)
        if q.dtype == torch.bfloat16:
            tol[b] += back((2.0 ** -10 * (1 + 2.0 ** -10) + m * 2.0 ** -35) * big.expand(-1, t.shape[1]))
    if q.dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * ref.abs()
    return ref, tol


def _check(got, q, pk, pv, kvs, lens):
    ref, tol = _reference(q, pk, pv, kvs, lens)
    err = (got.double() - ref).abs()
    assert bool((err <= tol).all()), f"worst {float(err.max()):.3g}, {float((err / tol).max()):.3g} of the bound"
    return float(err.max())


CASES = [  # hd, H, G, prefix, lens, n, window of the sequences' ring
    (128, 4, 4, 200, [0], 1, 128),
    (128, 4, 4, 1, [1, 0], 1, 128),
    (64, 8, 1, 63, [63, 5, 64], 2, 128),
    (64, 8, 2, 64, [64, 0, 127, 200], 3, 128),
    (32, 4, 4, 65, [31, 33], 4, 128),
    (32, 6, 2, 0, [7, 300], 1, 128),
    (128, 3, 3, 1000, [100] * 5, 1, 128),          # 5 rows a kv head
    (64, 32, 4, 517, [3, 90], 5, 128),             # 80 rows a kv head: the last tile in part
    (64, 32, 4, 2000, [33, 0, 64, 129], 2, 128),   # 64 rows
    (128, 2, 1, 1300, [20, 65], 65, 128),          # a chunk of each of two sequences
    (128, 2, 2, 130, [0] * 70, 1, 128),            # 70 rows, one a sequence
    (32, 8, 1, 4100, [700, 1, 64, 2], 9, 128),
    (128, 7, 1, 3000, [5, 6, 7, 8, 9], 1, 192),    # 35 rows: an odd group
    (64, 2, 2, 250, [130, 0], 129, 192),
    (128, 1, 1, 777, [10] * 33, 1, 128),           # 33 rows
    (64, 5, 5, 96, [1000, 3], 1, 128),             # own text longer than what is shared
    (128, 4, 4, 300, [600], 1, 128),               # eight waves to a kv head's own text
    (64, 8, 2, 100, [1000, 30], 2, 128),
    (64, 71, 1, 300, [200, 0], 1, 128),            # many query heads a kv head
    (128, 128, 1, 130, [33], 2, 128),
    (32, 34, 17, 64, [64, 0, 65], 7, 128),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"hd{c[0]}h{c[1]}-{c[2]}p{c[3]}b{len(c[4])}n{c[5]}")
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_shared(case, dtype):
    hd, H, G, P, lens, n, window = case
    rng = np.random.default_rng(P + n + hd)
    log(f"shared {case} {dtype}")
    prefix, pk, pv = _prefix(rng, hd, G, P, layer=1)
    kv = _cache(_shape(hd, H, G), len(lens), (max(lens) + n + 63) // 64 * 64, window)
    kvs = _fill(kv, rng, lens, n, G, hd, layer=1)
    q = _queries(rng, (len(lens), n, H, hd), dtype)
    worst = _check(_attend(prefix, kv, q, layer=1), q, pk, pv, kvs, lens)
    assert kv.read_state()["status"] == 0 and prefix.read_state()["status"] == 0
    log(f"worst error {worst:.3g}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hd,H,G,P,B,n", [(128, 4, 1, 30011, 3, 1), (64, 4, 2, 20000, 40, 2), (128, 2, 2, 9000, 150, 1),
                                          (64, 16, 1, 5555, 9, 7), (32, 2, 1, 70000, 1, 1), (128, 1, 1, 2111, 3, 300)])
def test_long_prefixes_and_many_rows(hd, H, G, P, B, n, dtype):
    rng = np.random.default_rng(P)
    log(f"shared long hd={hd} H={H} G={G} P={P} B={B} n={n} {dtype}")
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    lens = [int(x) for x in rng.integers(0, 150, B)]
    kv = _cache(_shape(hd, H, G, 1), B, 512, 384)
    kvs = _fill(kv, rng, lens, n, G, hd)
    q = _queries(rng, (B, n, H, hd), dtype)
    log(f"worst error {_check(_attend(prefix, kv, q), q, pk, pv, kvs, lens):.3g}")


# many rows, cut as the largest calls are: hd, H, G, P, B, n
MANY = [(64, 16, 8, 300, 8, 35),    # own texts: a wave's rows are its own
        (128, 8, 4, 200, 18, 67),
        (32, 12, 6, 1000, 11, 50),
        (128, 64, 32, 700, 8, 128),  # and the prefix's
        (64, 64, 64, 500, 4, 512)]


@pytest.mark.parametrize("case", MANY, ids=lambda c: f"hd{c[0]}h{c[1]}-{c[2]}p{c[3]}b{c[4]}n{c[5]}")
def test_many_sequences_of_many_rows(case):
    hd, H, G, P, B, n = case
    rng = np.random.default_rng(P + n)
    log(f"shared many {case}")
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    lens = [int(x) for x in rng.integers(0, 150, B)]
    lens[0] = 0
    kv = _cache(_shape(hd, H, G, 1), B, 704, (n + 63 + 63) // 64 * 64)
    kvs = _fill(kv, rng, lens, n, G, hd)
    q = _queries(rng, (B, n, H, hd), "bf16")
    log(f"worst error {_check(_attend(prefix, kv, q), q, pk, pv, kvs, lens):.3g}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,n,G", [(1, 7, 2), (3, 40, 2), (20, 40, 4)])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_bad_rows_that_are_not_seen(hd, B, n, G, dtype):
    """NaN and infinities in K and V rows of the newest: the queries that see them, and no others."""
    torch = torch_cuda()
    rng = np.random.default_rng(hd + n + B)
    group, P = 2, 100
    H, L = group * G, 77
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    kv = _cache(_shape(hd, H, G, 1), B, 192, 128)
    kvs = _fill(kv, rng, [L] * B, n, G, hd)
    q = _queries(rng, (B, n, H, hd), dtype)
    log(f"bad rows not seen hd={hd} B={B} n={n} {dtype}")
    clean = _attend(prefix, kv, q)
    _check(clean, q, pk, pv, kvs, [L] * B)
    k, v = (np.stack([kvs[b][i][L:] for b in range(B)]) for i in range(2))
    first, nan, key = n // 3, n // 2, 2 * n // 3
    v[:, first, 0, 5], v[:, nan, 0, 6], k[:, key, 1, 2] = np.inf, np.nan, np.nan
    binding.specdec_kv_append(kv, 0, _bf16(k), _bf16(v))
    got = _attend(prefix, kv, q)
    _check(got[:, :first], q[:, :first], pk, pv, kvs, [L] * B)
    h0, h1 = got[:, :, :group], got[:, :, group:2 * group]
    assert (h0[:, first:, :, 5] == float("inf")).all() or not torch.isfinite(h0[:, first:, :, 5]).any()
    assert torch.isfinite(h0[:, :nan, :, 6]).all() and torch.isnan(h0[:, nan:, :, 6]).all()
    assert torch.isfinite(h1[:, :key]).all() and torch.isnan(h1[:, key:]).all()
    got[:, first:, :group, 5], got[:, nan:, :group, 6] = clean[:, first:, :group, 5], clean[:, nan:, :group, 6]
    got[:, key:, group:2 * group] = clean[:, key:, group:2 * group]
    _check(got, q, pk, pv, kvs, [L] * B)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("B", [1, 40])
@pytest.mark.parametrize("P,L", [(0, 0), (30, 0), (0, 70)])
def test_each_key_in_turn_is_nan(hd, B, P, L):
    """A NaN key among the newest of many rows: what one query sees leaves the maxima of the others', of
    other tiles, alone; also where those have seen nothing before."""
    torch = torch_cuda()
    rng = np.random.default_rng(hd + B)
    G, H, n = 2, 4, 40
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    kv = _cache(_shape(hd, H, G, 1), B, 128, 128)
    kvs = _fill(kv, rng, [L] * B, n, G, hd)
    q = _queries(rng, (B, n, H, hd), "bf16")
    ref, tol = _reference(q, pk, pv, kvs, [L] * B)
    k, v = (np.stack([kvs[b][i][L:] for b in range(B)]) for i in range(2))
    for at in range(0, n, 3):
        bad = k.copy()
        bad[:, at] = np.nan
        binding.specdec_kv_append(kv, 0, _bf16(bad), _bf16(v))
        got = _attend(prefix, kv, q).double()
        assert bool(((got - ref).abs() <= tol)[:, :at].all()), (hd, B, P, L, at)
        assert bool(torch.isnan(got[:, at:]).all())


# Own texts that are cut over workgroups: hd, H, G, P, lens, n
LONG = [(128, 2, 2, 300, [20000], 1), (128, 2, 1, 100, [9000, 17000, 300], 20), (64, 4, 2, 500, [40000, 7], 5),
        (128, 2, 1, 700, [9000, 0], 70), (32, 8, 2, 64, [30000, 33000, 5, 20000], 3), (64, 2, 2, 0, [30000], 100),
        (128, 32, 32, 500, [9000] * 3, 1)]


@pytest.mark.parametrize("case", LONG, ids=lambda c: f"hd{c[0]}h{c[1]}-{c[2]}b{len(c[4])}n{c[5]}")
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_own_texts(case, dtype):
    hd, H, G, P, lens, n = case
    rng = np.random.default_rng(P + n)
    log(f"shared, long own texts {case} {dtype}")
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    kv = _cache(_shape(hd, max(H, 2 * G), G, 1), len(lens), (max(lens) + n + 63) // 64 * 64, 192)
    kvs = _fill(kv, rng, lens, n, G, hd)
    q = _queries(rng, (len(lens), n, H, hd), dtype)
    ws = binding.shared_attention_workspace(prefix, kv, H, n, q.dtype)
    for _ in range(3):  # (counters of the parts are back at zero)
        _check(_attend(prefix, kv, q, ws=ws), q, pk, pv, kvs, lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 70])
def test_magnitudes(dtype, n):
    """Heads of unlike magnitudes (scales far from 1), scores that leave one key, and flat ones."""
    rng = np.random.default_rng(n)
    hd, G, H, P, lens = 64, 3, 6, 900, [70, 3]
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1, spread=True)
    kv = _cache(_shape(hd, H, G, 1), 2, 192, 192)
    kvs = _fill(kv, rng, lens, n, G, hd, spread=True)
    for sigma in (1e-3, 1.0, 100.0):
        q = _queries(rng, (2, n, H, hd), dtype, sigma)
        log(f"magnitudes n={n} {dtype} sigma {sigma}")
        _check(_attend(prefix, kv, q), q, pk, pv, kvs, lens)


@pytest.mark.parametrize("n,H", [(1, 2), (40, 4)])
def test_without_a_prefix_it_is_the_plain_attention(n, H):
    torch = torch_cuda()
    rng = np.random.default_rng(1)
    hd, G, lens = 128, 2, [500, 0, 64]
    prefix, _, _ = _prefix(rng, hd, G, 0, n_layers=1)
    kv = _cache(_shape(hd, H, G, 1), 3, 640, 128)
    kvs = _fill(kv, rng, lens, n, G, hd)
    q = _queries(rng, (3, n, H, hd), "f32")
    none = np.zeros((0, G, hd))
    plain = torch.empty_like(q)
    binding.specdec_attention(kv, 0, q, plain)  # (sums of another order: both within the bound)
    _check(plain, q, none, none, kvs, lens)
    _check(_attend(prefix, kv, q), q, none, none, kvs, lens)
    # an empty prefix under a host bound of its whole capacity
    big = _cache(_shape(hd, G, G, 1), 2, 4096)
    big.set_state([0, 0], [[0, 1]] * 2, [1] * 2)
    big.kv.len_upper = 4096
    ws = binding.shared_attention_workspace(big, kv, H, n)
    ws.fill_(255)
    _check(_attend(big, kv, q, ws=ws), q, none, none, kvs, lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P,n", [(70, 1), (1000, 3), (1000, 30), (4032, 1)])
def test_a_host_bound_above_the_length(P, n, dtype):
    """Parts that the prefix does not reach are neither written nor read; a workspace of NaN."""
    rng = np.random.default_rng(P + n)
    hd, H, G, lens = 64, 8, 2, [10, 200]
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1, cap=8192)
    prefix.kv.len_upper = 8192
    kv = _cache(_shape(hd, H, G, 1), 2, 1024, 128)
    kvs = _fill(kv, rng, lens, n, G, hd)
    kv.kv.len_upper = 1024 - n
    q = _queries(rng, (2, n, H, hd), dtype)
    ws = binding.shared_attention_workspace(prefix, kv, H, n, q.dtype)
    ws.fill_(255)
    log(f"bound above the length P={P} n={n} {dtype}")
    _check(_attend(prefix, kv, q, ws=ws), q, pk, pv, kvs, lens)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 50])
def test_a_host_bound_below_the_length(n, dtype):
    """The prefix counts up to the host's bound, and the cache's status says so."""
    rng = np.random.default_rng(n)
    hd, H, G, lens = 64, 2, 2, [10, 20]
    prefix, pk, pv = _prefix(rng, hd, G, 300, n_layers=1)
    prefix.kv.len_upper = 192
    kv = _cache(_shape(hd, H, G, 1), 2, 128, 128)
    kvs = _fill(kv, rng, lens, n, G, hd)
    q = _queries(rng, (2, n, H, hd), dtype)
    log(f"bound below the length n={n} {dtype}")
    _check(_attend(prefix, kv, q), q, pk[:192], pv[:192], kvs, lens)
    assert kv.read_state()["status"] == -3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("at", [5, 700, 1030])
def test_bad_rows_of_a_prefix(at, n, dtype):
    """A NaN key makes every row of its kv head NaN, a bad value its dim of them, in codes (at 5, 700)
    and in the ring (1030); the other kv heads do not change."""
    torch = torch_cuda()
    rng = np.random.default_rng(at + n)
    hd, H, G, P, lens = 64, 6, 3, 1040, [9, 100]
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    kv = _cache(_shape(hd, H, G, 1), 2, 192, 128)
    kvs = _fill(kv, rng, lens, n, G, hd)
    q = _queries(rng, (2, n, H, hd), dtype)
    log(f"bad rows at {at} n={n} {dtype}")
    clean = _attend(prefix, kv, q)
    _check(clean, q, pk, pv, kvs, lens)
    k, v = pk.copy(), pv.copy()
    k[at, 0, 3] = np.nan
    v[at, 1, 7], v[at, 1, 9] = np.nan, np.inf
    lo = at // 64 * 64  # (the other rows of that block are stored values: they stay)
    prefix.write_context(0, 1, lo, _bf16(k[lo:]), _bf16(v[lo:]))
    got = _attend(prefix, kv, q)
    group = H // G
    assert torch.isnan(got[:, :, :group]).all()
    bad = got[:, :, group:2 * group]
    assert torch.isnan(bad[..., 7]).all() and not torch.isfinite(bad[..., 9]).any()
    keep = [d for d in range(hd) if d not in (7, 9)]
    assert torch.equal(bad[..., keep], clean[:, :, group:2 * group][..., keep])
    assert torch.equal(got[:, :, 2 * group:], clean[:, :, 2 * group:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 70])
@pytest.mark.parametrize("where", ["prefix", "own", "codes of the prefix"])
def test_scores_below_float32(where, n, dtype):
    """Keys whose score is below float32's range weigh nothing, also where one of the sets has no others."""
    rng = np.random.default_rng(n)
    hd, H, G, P, lens = 64, 2, 1, 500, [100]
    rows = lambda m: [rng.normal(0, 1.3, (m, G, hd)) for _ in range(2)]  # noqa: E731
    (pk, pv), (k, v) = rows(P), rows(100 + n)
    for x in (pk, k):
        x[:, :, 0] = 0
    low = {"prefix": pk, "own": k, "codes of the prefix": pk[:448]}[where]
    low[:] = 0
    low[:, :, 0] = -2.0 ** 118
    pk, pv, k, v = (_np(_bf16(x)) for x in (pk, pv, k, v))
    prefix, kv = _cache(_shape(hd, G, G, 1), 1, 512), _cache(_shape(hd, H, G, 1), 1, 192, 192)
    prefix.write_context(0, 0, 0, _bf16(pk), _bf16(pv))
    prefix.set_state([P], [[0, 1]], [1])
    kv.write_context(0, 0, 0, _bf16(k[:100]), _bf16(v[:100]))
    kv.set_state([100], [[0, 1]], [1])
    binding.specdec_kv_append(kv, 0, _bf16(k[None, 100:]), _bf16(v[None, 100:]))
    q = _queries(rng, (1, n, H, hd), dtype)
    q[..., 0] = 2.0 ** 14
    log(f"scores below float32: {where} n={n} {dtype}")
    got = _attend(prefix, kv, q, at=0)
    q[..., 0] = 0
    pk, pv = fp8.stored(pk, 448), fp8.stored(pv, 448)
    own = [fp8.stored(k, 64), fp8.stored(v, 64)]
    if where == "own":
        ref, tol = _reference(q, pk, pv, [[x[:0] for x in own]], [P + 1000])  # (no row of its own is seen)
    else:
        cut = slice(448, P) if where[0] == "c" else slice(0, 0)
        ref, tol = _reference(q, pk[cut], pv[cut], [own], lens)
    assert bool(((got.double() - ref).abs() <= tol).all())


def test_in_place_and_other_streams():
    """out may be q; a call on another stream than the current one, its own workspace."""
    torch = torch_cuda()
    rng = np.random.default_rng(2)
    hd, H, G, P, lens, n = 128, 8, 2, 1111, [4, 50, 0], 3
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    kv = _cache(_shape(hd, H, G, 1), 3, 128, 128)
    kvs = _fill(kv, rng, lens, n, G, hd)
    side = torch.cuda.Stream()
    for dtype in ("f32", "bf16"):
        q = _queries(rng, (3, n, H, hd), dtype)
        want = _attend(prefix, kv, q)
        _check(want, q, pk, pv, kvs, lens)
        out = q.clone()
        binding.specdec_attention_shared(prefix, kv, 0, out, out, prefix_b=1)
        assert torch.equal(out, want)
        out = torch.full_like(q, float("nan"))
        side.wait_stream(torch.cuda.current_stream())
        binding.specdec_attention_shared(prefix, kv, 0, q, out, prefix_b=1, stream=side)
        side.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_prefix_for_two_batches_at_once(dtype):
    """Two caches' calls on two streams over one prefix, eager and captured, replayed several times."""
    torch = torch_cuda()
    rng = np.random.default_rng(3)
    hd, H, G, P, n = 64, 8, 1, 6000, 2
    prefix, pk, pv = _prefix(rng, hd, G, P, n_layers=1)
    lens = [[300, 17], [33, 48]]
    kvs = [_cache(_shape(hd, H, G, 1), 2, 320, 128) for _ in lens]
    held = [_fill(kv, rng, x, n, G, hd) for kv, x in zip(kvs, lens)]
    q = [_queries(rng, (2, n, H, hd), dtype) for _ in lens]
    out = [torch.empty_like(x) for x in q]
    ws = [binding.shared_attention_workspace(prefix, kv, H, n, q[0].dtype) for kv in kvs]
    streams, graphs = [torch.cuda.Stream() for _ in lens], []
    torch.cuda.synchronize()
    for j in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[j]):
            binding.specdec_attention_shared(prefix, kvs[j], 0, q[j], out[j], ws[j], 1)
        graphs.append(g)
    for rep in range(4):
        for o in out:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        log(f"one prefix, two batches, {rep} {dtype}")
        for _ in range(5):
            for j in range(2):
                if rep % 2:
                    binding.specdec_attention_shared(prefix, kvs[j], 0, q[j], out[j], ws[j], 1, stream=streams[j])
                else:
                    with torch.cuda.stream(streams[j]):
                        graphs[j].replay()
        torch.cuda.synchronize()
        for j in range(2):
            _check(out[j], q[j], pk, pv, held[j], lens[j])


def test_a_prefix_past_four_gib():
    """The last sequence of a prefix cache whose codes take more than 2^32 bytes, in its last layer."""
    rng = np.random.default_rng(4)
    hd, H, G, P = 128, 4, 4, 4090
    prefix, pk, pv = _prefix(rng, hd, G, P, batch=300, at=299, n_layers=4, layer=3)
    assert 4 * 300 * G * 2 * 4096 * hd > 2 ** 32
    kv = _cache(_shape(hd, H, G, 4), 2, 128, 128)
    kvs = _fill(kv, rng, [3, 60], 1, G, hd, layer=3)
    for dtype in ("f32", "bf16"):
        q = _queries(rng, (2, 1, H, hd), dtype)
        _check(_attend(prefix, kv, q, layer=3, at=299), q, pk, pv, kvs, [3, 60])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_decode_loop(dtype):
    """The attention block of a model with head norms, as it is served: a prompt's chunk, then tokens one
    by one in a captured graph, over a prefix that two requests share, against 64 bits over the
    rows that the caches hold; those against the oracle's norm and rotation."""
    torch = torch_cuda()
    rng = np.random.default_rng(5)
    hd, H, G, P, B, chunk = 64, 8, 2, 333, 2, 100
    gains = [f32(1 + rng.normal(0, 0.2, hd)) for _ in range(2)]
    r = binding.Rope(hd, q_gain=gains[0], k_gain=gains[1], eps=1e-5)
    freq = rope_oracle.freqs(hd, 10000.0)
    turned = lambda x, first, g: rope_oracle.apply(  # noqa: E731
        _np(x), first + np.arange(x.shape[1])[None], freq, False, _np(gains[g]), 1e-5)
    rows = lambda b, n: [f32(rng.normal(0, 1.3, (b, n, h, hd))) for h in (H, G, G)]  # noqa: E731
    # (norm and rotation: 16.1 2^-24 of at most two normalised values below sqrt(hd) times a gain below 2)
    near = 16.1 * 2.0 ** -24 * 2 * 2 * hd ** 0.5

    prefix = _cache(_shape(hd, H, G, 1), 1, 384, 448)
    q, k, v = rows(1, P)
    binding.specdec_rope_append(prefix, 0, r, q, k, v, torch.empty_like(q))
    want = turned(k, 0, 1)[0]
    err = np.abs(_np(prefix.read_context(0, 0, 0, P)[0]) - want)
    assert (err <= near + 2.0 ** -8 * np.abs(want)).all()
    binding.specdec_kv_advance(prefix, P)
    pk, pv = (_np(t) for t in prefix.read_context(0, 0, 0, P))

    kv = _cache(_shape(hd, H, G, 1), B, 256, 192)
    typed = lambda n: torch.empty((B, n, H, hd), dtype=_queries(rng, 1, dtype).dtype, device="cuda")  # noqa: E731

    def check(new, qr, out, now):
        n = qr.shape[1]
        want = turned(new[0], P + now, 0)
        assert (np.abs(_np(qr) - want) <= near + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)).all()
        held = [[_np(t) for t in kv.read_context(0, b, 0, now + n)] for b in range(B)]
        want = turned(new[1], P + now, 1)
        for b in range(B):
            assert (np.abs(held[b][0][now:] - want[b]) <= near + 2.0 ** -8 * np.abs(want[b])).all()
            np.testing.assert_array_equal(held[b][1][now:], _np(new[2][b].to(torch.bfloat16)))
        _check(out, qr, pk, pv, held, [now] * B)

    new, qr, out = rows(B, chunk), typed(chunk), typed(chunk)
    binding.specdec_rope_append(kv, 0, r, *new, qr, offset=P)
    binding.specdec_attention_shared(prefix, kv, 0, qr, out)
    check(new, qr, out, 0)
    binding.specdec_kv_advance(kv, chunk)

    new, qr, out = rows(B, 1), typed(1), typed(1)
    ws = binding.shared_attention_workspace(prefix, kv, H, 1, qr.dtype)
    kv.kv.len_upper = chunk + 10  # (what the last replay reaches)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.specdec_rope_append(kv, 0, r, *new, qr, offset=P)
        binding.specdec_attention_shared(prefix, kv, 0, qr, out, ws)
        binding.specdec_kv_advance(kv, 1)
    for i in range(8):
        for t, x in zip(new, rows(B, 1)):
            t.copy_(x)
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        log(f"decode loop {dtype}, token {i}")
        check(new, qr, out, chunk + i)  # (no block is completed: the new row is still as it was appended)
    state = kv.read_state()
    assert state["status"] == 0 and (state["len"] == chunk + 8).all()
