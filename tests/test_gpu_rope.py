"""Norm and rotation of queries and keys, alone and into an 8-bit cache, against the float64 oracle.

The bound.  With y the normalised value, a pair's result y_a c - y_b s in float32: a sum of squares
is 2 roundings of a pair and 6 levels of sums at most, the mean with eps one more (9 steps of 2^-24, 4.5 of its
square root), the factor 1 / sqrt within 2^-23 (2 steps), its product and the gain's two more:
8.5 steps of y; the angle, reduced in float64 to at most half a turn, enters as a float32 of at most 1 in half
turns (half a step, 2^-25, times pi), the functions are within 4 units in the last place (2^-24 of
1 each), products and sum are two roundings:
  |out - ref| <= (8.5 + 2 + pi / 2 + 4) 2^-24 (|y_a| + |y_b|) < 16.1 2^-24 (|y_a| + |y_b|)
and the angle itself, position times frequency in float64 on both sides, up to 8 roundings of
2^-53 of it.  Results of 16 bits: half a step, 2^-8 of the value, more.  Below float32's normal values
a rounding is half a step of 2^-149, eight of them at most.
"""
import numpy as np
import pytest

from oracle import rope as oracle
from paper_2608_10362_amd import binding
from tests.gpu_util import f32, i32, log, torch_cuda
from tests.test_gpu_fp8_cache import _cache, _np, _shape

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _type(name):
    torch = torch_cuda()
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _t(x, name="f32"):
    return f32(x).to(_type(name))


def _tol(x, pos, freq, interleaved, gain, eps, out):
    y = oracle.norm(x, gain, eps)
    a, b = oracle.pairs(2 * len(freq), interleaved)
    size = np.abs(y)
    both = size[..., a] + size[..., b]
    angle = np.abs(np.asarray(pos, np.float64))[:, :, None, None] * freq
    tol = 8.5 * 2.0 ** -24 * size
    tol[..., a] = tol[..., b] = (16.1 * 2.0 ** -24 + 8 * 2.0 ** -53 * angle) * both
    ref = oracle.rotate(y, pos, freq, interleaved)
    return ref, tol * (1 + 2.0 ** -8) + (2.0 ** -8 * np.abs(ref) if out == "bf16" else 0.0)


def _compare(got, x, pos, freq, interleaved, gain, eps, out):
    ref, tol = _tol(x, pos, freq, interleaved, gain, eps, out)
    err = np.abs(_np(got).astype(np.float64) - ref)
    assert (err <= tol + 2.0 ** -147).all(), f"{(err - tol).max():.3g} past the bound, worst {err.max():.3g}"
    return float((err / np.maximum(tol, 1e-300)).max())


def _inputs(rng, B, n, H, G, hd, dtype, fused=True, lead=0):
    """q, k, v as views of one buffer of rows (`lead` elements before the first), or on their own."""
    torch = torch_cuda()
    if not fused:
        return [_t(rng.normal(0, 1.3, (B, n, h, hd)), dtype) for h in (H, G, G)]
    width = (H + 2 * G) * hd + 3 * (lead > 0)
    buf = _t(rng.normal(0, 1.3, lead + B * n * width), dtype)
    rows = torch.as_strided(buf, (B, n, (H + 2 * G) * hd), (n * width, width, 1), lead)
    return [x.unflatten(-1, (-1, hd)) for x in rows.split([H * hd, G * hd, G * hd], -1)]


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", [
    # batch, n, heads, kv heads, rotary share of the head (16: 16 dims), norms, lead, offset
    (1, 1, 4, 4, 1, "qk", 0, 4095), (3, 7, 5, 1, 0.5, "qk", 1, 0), (2, 9, 32, 4, 16, "", 0, 131072),
    (5, 1, 1, 1, 1, "q", 3, 7), (1, 130, 3, 2, 1, "k", 0, 0), (2, 3, 71, 3, 0, "qk", 5, 100)],
    ids=lambda c: f"b{c[0]}n{c[1]}h{c[2]}-{c[3]}r{c[4]}{c[5]}")
def test_apply(hd, dtype, out, interleaved, case):
    B, n, H, G, share, norms, lead, offset = case
    rng = np.random.default_rng(hd + n + H)
    rot = share if share == 16 else int(hd * share)
    log(f"rope apply hd={hd} {dtype}->{out} interleaved={interleaved} {case}")
    q, k, _ = _inputs(rng, B, n, H, G, hd, dtype, lead=lead)
    gq, gk = (_t(1 + rng.normal(0, 0.2, hd), dtype) if s in norms else None for s in "qk")
    r = binding.Rope(hd, rotary_dim=rot, interleaved=interleaved, q_gain=gq, k_gain=gk, eps=EPS)
    torch = torch_cuda()
    q_out, k_out = (torch.full(x.shape, float("nan"), dtype=_type(out), device="cuda") for x in (q, k))
    pos = rng.integers(-5, 1000000, (B, n)).astype(np.int32) if n != 7 else None
    binding.specdec_rope_apply(r, q, k, q_out, k_out, positions=None if pos is None else i32(pos), offset=offset)
    pos = (np.broadcast_to(np.arange(n), (B, n)) if pos is None else pos).astype(np.int64) + offset
    freq = oracle.freqs(rot, 10000.0)
    worst = 0
    for got, x, g in ((q_out, q, gq), (k_out, k, gk)):
        worst = max(worst, _compare(got, _np(x), pos, freq, interleaved, None if g is None else _np(g), EPS, out))
    log(f"worst {worst:.3g} of the bound")


def test_own_frequencies_and_far_positions():
    rng = np.random.default_rng(0)
    hd, B, n = 64, 2, 5
    q, k, _ = _inputs(rng, B, n, 3, 1, hd, "f32")
    freq = np.exp(rng.uniform(np.log(1e-6), np.log(3.0), 16))
    r = binding.Rope(hd, rotary_dim=32, freqs=freq)
    pos = np.array([[0, 1, -1, 2 ** 31 - 1, -2 ** 31], [10 ** 6, 10 ** 7, 123456789, 65536, 3]], np.int32)
    q_out, k_out = torch_cuda().empty_like(q.contiguous()), torch_cuda().empty_like(k.contiguous())
    for offset in (0, 2 ** 33 + 5):
        binding.specdec_rope_apply(r, q, k, q_out, k_out, positions=i32(pos), offset=offset)
        for got, x in ((q_out, q), (k_out, k)):
            _compare(got, _np(x), pos.astype(np.int64) + offset, freq, False, None, 0.0, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_one_of_the_two(dtype):
    """Outputs over their own inputs, in a fused buffer too; queries alone, keys alone; a strided output."""
    torch = torch_cuda()
    rng = np.random.default_rng(3)
    hd, B, n, H, G = 64, 2, 21, 6, 2
    for fused in (False, True):
        q, k, v = _inputs(rng, B, n, H, G, hd, dtype, fused)
        g = _t(1 + rng.normal(0, 0.2, hd), dtype)
        r = binding.Rope(hd, q_gain=g, k_gain=g, eps=EPS)
        want_q, want_k = (torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (q, k))
        binding.specdec_rope_apply(r, q, k, want_q, want_k)
        only = torch.zeros_like(want_q)
        binding.specdec_rope_apply(r, q, None, only, None)
        assert torch.equal(only, want_q)
        wide = torch.zeros((B, n, G * hd + 40), dtype=q.dtype, device="cuda")
        binding.specdec_rope_apply(r, None, k, None, wide[..., 8:8 + G * hd].unflatten(-1, (G, hd)))
        assert torch.equal(wide[..., 8:8 + G * hd].unflatten(-1, (G, hd)), want_k)
        assert not wide[..., :8].any() and not wide[..., 8 + G * hd:].any()
        held = v.clone()
        binding.specdec_rope_apply(r, q, k, q, k)
        assert torch.equal(q, want_q) and torch.equal(k, want_k) and torch.equal(v, held)


def test_values_at_the_edges():
    """Magnitudes whose squares float32 does not hold; a zero row; NaN and infinities stay in their head."""
    torch = torch_cuda()
    rng = np.random.default_rng(4)
    hd, n, H = 32, 2, 9
    x = rng.normal(0, 1, (1, n, H, hd)).astype(np.float32)
    x[:, :, 1] *= 2.0 ** 120
    x[:, :, 2] *= 2.0 ** -120
    x[:, :, 3] = 0
    x[0, 0, 4, 3] = np.nan
    x[0, 1, 5, 3] = np.inf
    x[:, :, 6] *= 2.0 ** 60
    x[:, :, 7] *= 2.0 ** -140  # (no longer normal)
    for eps in (0.0, EPS):
        r = binding.Rope(hd, q_gain=f32(np.ones(hd)), eps=eps)
        out = torch.empty((1, n, H, hd), device="cuda")
        binding.specdec_rope_apply(r, f32(x), None, out, None, offset=77)
        got, pos, freq = _np(out), np.array([[77, 78]]), oracle.freqs(hd, 10000.0)
        eps = float(np.float32(eps))
        fine = [0, 1, 2, 6, 7, 8] + ([3] if eps else [])
        _compare(out[:, :, fine], x[:, :, fine], pos, freq, False, np.ones(hd), eps, "f32")
        assert eps or np.isnan(got[:, :, 3]).all()  # (0 / 0)
        assert np.isnan(got[0, 0, 4]).all()
        # an infinity: 0 for the finite entries, NaN for itself and its pair's other dim
        rest = [d for d in range(hd) if d not in (3, 19)]
        assert np.isnan(got[0, 1, 5, [3, 19]]).all() and (got[0, 1, 5, rest] == 0).all()
        _compare(out[:, 1:, 4:5], x[:, 1:, 4:5], pos[:, 1:], freq, False, np.ones(hd), eps, "f32")


def _ring_rows(kv, layer, lens, n):
    return [[_np(x) for x in kv.read_context(layer, b, L, n)] for b, L in enumerate(lens)]


@pytest.mark.parametrize("hd,H,G", [(32, 6, 2), (64, 32, 4), (128, 3, 3), (128, 5, 1), (64, 9, 9)])
@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("lens,n,window", [([0], 1, 128), ([63, 64, 5, 127, 200], 1, 128), ([7, 120, 0, 1], 5, 128),
                                           ([3, 90], 65, 128), ([0, 8, 250], 129, 192), ([100], 8, 128)])
def test_append(hd, H, G, dtype, out, lens, n, window):
    """The cache's rows and the queries, for rows anywhere in the ring; the rows before them, other
    sequences' places and the other layer stay as they were."""
    torch = torch_cuda()
    rng = np.random.default_rng(hd + n + len(lens))
    B = len(lens)
    cap = (max(lens) + n + 63) // 64 * 64
    log(f"rope append hd={hd} H={H} G={G} {dtype}->{out} lens={lens} n={n}")
    kv, plain = _cache(_shape(hd, H, G), B, cap, window), _cache(_shape(hd, H, G), B, cap, window)
    gq, gk = _t(1 + rng.normal(0, 0.2, hd), dtype), _t(1 + rng.normal(0, 0.2, hd), dtype)
    r = binding.Rope(hd, rotary_dim=hd if n != 5 else 16, interleaved=n == 8, q_gain=gq, k_gain=gk, eps=EPS)
    for b, L in enumerate(lens):
        if L:
            k, v = (_t(rng.normal(0, 1.3, (L, G, hd)), "bf16") for _ in range(2))
            for c in (kv, plain):
                c.write_context(0, b, 0, k, v)
                c.write_context(1, b, 0, v, k)
    for c in (kv, plain):
        c.set_state(lens, [[0, 1]] * B, [1] * B)
    q, k, v = _inputs(rng, B, n, H, G, hd, dtype, lead=3 if n == 5 else 0)
    q_out = torch.full((B, n, H, hd), float("nan"), dtype=_type(out), device="cuda")
    binding.specdec_rope_append(kv, 1, r, q, k, v, q_out, offset=1000)
    pos = np.array(lens)[:, None] + np.arange(n) + 1000
    freq = oracle.freqs(r.c.rotary_dim, 10000.0)
    _compare(q_out, _np(q), pos, freq, n == 8, _np(gq), EPS, out)
    rows = _ring_rows(kv, 1, lens, n)
    for b in range(B):
        ref, tol = _tol(_np(k)[b:b + 1], pos[b:b + 1], freq, n == 8, _np(gk), EPS, "bf16")
        assert (np.abs(rows[b][0] - ref[0]) <= tol[0]).all()
        np.testing.assert_array_equal(rows[b][1], _np(v[b].to(torch.bfloat16)))
    # the same rows put there by specdec_kv_append leave the same bytes everywhere
    k_out = torch.empty((B, n, G, hd), dtype=torch.bfloat16, device="cuda")
    binding.specdec_rope_apply(r, None, k, None, k_out, positions=i32(pos))
    binding.specdec_kv_append(plain, 1, k_out, v.to(torch.bfloat16).contiguous())
    assert torch.equal(kv.data, plain.data)
    # given positions
    binding.specdec_rope_append(kv, 1, r, q, k, v, q_out, positions=i32(pos - 1000), offset=1000)
    assert torch.equal(kv.data, plain.data)
    assert kv.read_state()["status"] == 0


def test_append_past_the_capacity_sets_the_status():
    """A host bound that is too low: rows past the capacity are not stored, their queries are."""
    torch = torch_cuda()
    rng = np.random.default_rng(8)
    hd, H, G, n = 64, 2, 1, 9
    kv = _cache(_shape(hd, H, G), 2, 128, 128)
    kv.set_state([128, 10], [[0, 1]] * 2, [1] * 2)
    kv.kv.len_upper = 10
    q, k, v = _inputs(rng, 2, n, H, G, hd, "f32")
    out, r = torch.full((2, n, H, hd), float("nan"), device="cuda"), binding.Rope(hd)
    before = kv.data.clone()
    binding.specdec_rope_append(kv, 0, r, q, k, v, out)
    assert kv.read_state()["status"] == -3
    _compare(out, _np(q), np.array([128, 10])[:, None] + np.arange(n), oracle.freqs(hd, 10000.0), False, None, 0, "f32")
    np.testing.assert_array_equal(_np(kv.read_context(0, 1, 10, n)[1]), _np(v[1].to(torch.bfloat16)))
    # (nothing of the first sequence's ring changed)
    skip = 2 * G * 4 * 128 * 4
    ring = 2 * 128 * hd * 2
    assert torch.equal(kv.data[skip:skip + ring], before[skip:skip + ring])


def test_streams_and_graphs():
    """On another stream than the current one; captured, and replayed at lengths that grew."""
    torch = torch_cuda()
    rng = np.random.default_rng(9)
    hd, H, G, n, B = 64, 8, 2, 3, 2
    kv = _cache(_shape(hd, H, G, 1), B, 256, 128)
    lens = np.array([5, 60])
    kv.set_state(lens, [[0, 1]] * B, [1] * B)
    r = binding.Rope(hd, q_gain=f32(1 + rng.normal(0, 0.2, hd)), eps=EPS)
    q, k, v = _inputs(rng, B, n, H, G, hd, "bf16")
    out = torch.empty((B, n, H, hd), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    binding.specdec_rope_append(kv, 0, r, q, k, v, out, stream=side)
    side.synchronize()
    freq, gain = oracle.freqs(hd, 10000.0), _np(r.gains[0])
    check = lambda: _compare(out, _np(q), lens[:, None] + np.arange(n), freq, False, gain, EPS, "f32")  # noqa: E731
    check()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.specdec_rope_append(kv, 0, r, q, k, v, out)
    for rep in range(4):
        out.fill_(float("nan"))
        q.copy_(_t(rng.normal(0, 1.3, q.shape), "bf16"))
        g.replay()
        torch.cuda.synchronize()
        check()
        binding.specdec_kv_advance(kv, n)
        lens = lens + n
        assert (kv.read_state()["len"] == lens).all()


def test_many_rows_and_the_largest_widths():
    """More rows than the card holds at once, and heads past one workgroup's."""
    torch = torch_cuda()
    rng = np.random.default_rng(10)
    for B, n, H, G, hd in ((1, 20011, 2, 1, 32), (700, 3, 128, 1, 128), (1, 2, 1024, 1024, 64)):
        q, k, _ = _inputs(rng, B, n, H, G, hd, "bf16", fused=False)
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        log(f"rows {B} x {n}, {H} and {G} heads of {hd}")
        binding.specdec_rope_apply(binding.Rope(hd), q, k, q_out, k_out)
        pos = np.broadcast_to(np.arange(n), (B, n))
        for got, x in ((q_out, q), (k_out, k)):
            _compare(got, _np(x), pos, oracle.freqs(hd, 10000.0), False, None, 0.0, "bf16")
