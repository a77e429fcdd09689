"""Refusals of the norm and rotation calls that launch nothing (no GPU needed)."""
import ctypes

import pytest

from paper_2608_10362_amd import binding

FAKE = 1 << 20  # never dereferenced: the calls fail first
r = ctypes.byref


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(binding.LIB_PATH):
        from paper_2608_10362_amd import build
        build.build()
    return binding.lib()


def _rope(lib, hd=64, rot=64):
    d = binding.RopeDesc()
    assert lib.specdec_rope_init(r(d), hd, rot, 10000.0, 0, FAKE, None, 1, 1e-5) == 0
    return d


def test_init(lib):
    d = _rope(lib, 64, 32)
    assert (d.head_dim, d.rotary_dim, d.interleaved, d.gain_dtype, d.q_gain, d.k_gain) == (64, 32, 0, 1, FAKE, None)
    for j in range(16):
        assert abs(d.freq[j] - 10000.0 ** (-j / 16)) < 1e-15
    assert not any(d.freq[16:])
    call = lambda hd=64, rot=64, base=1e4, inter=0, dt=0, eps=0.0: lib.specdec_rope_init(  # noqa: E731
        r(d), hd, rot, base, inter, None, None, dt, eps)
    assert call() == 0 and call(rot=0) == 0
    for bad in ({"hd": 96}, {"hd": 256}, {"rot": 8}, {"rot": 80}, {"rot": 24}):
        assert call(**bad) == -2, bad
    for bad in ({"hd": 0}, {"rot": -16}, {"base": 0.0}, {"base": float("nan")}, {"base": float("inf")}, {"inter": 2},
                {"dt": 2}, {"eps": -1.0}, {"eps": float("nan")}):
        assert call(**bad) == -1, bad
    assert lib.specdec_rope_init(None, 64, 64, 1e4, 0, None, None, 0, 0.0) == -1


def _apply(lib, rope, batch=2, n=3, H=4, G=2, dtype=0, q=FAKE, ld_q=256, k=FAKE << 1, ld_k=128, out_dtype=0,
           q_out=FAKE << 2, ld_qo=256, k_out=FAKE << 3, ld_ko=128):
    return lib.specdec_rope_apply(r(rope) if rope is not None else None, batch, n, H, G, dtype, q, ld_q, k, ld_k, None,
                                  0, out_dtype, q_out, ld_qo, k_out, ld_ko, None)


def test_apply(lib):
    d = _rope(lib)
    for bad in ({"batch": 0}, {"n": 0}, {"H": -1}, {"dtype": 2}, {"out_dtype": 3}, {"q": None}, {"q_out": None},
                {"H": 0}, {"k": None}, {"k_out": None}, {"G": 0}, {"ld_q": 255}, {"ld_k": 127}, {"ld_qo": 255},
                {"ld_ko": 127}, {"q": None, "k": None, "q_out": None, "k_out": None, "H": 0, "G": 0}):
        assert _apply(lib, d, **bad) == -1, bad
    assert _apply(lib, None) == -1
    assert _apply(lib, d, batch=1 << 15, n=1 << 10) == -2
    assert _apply(lib, d, H=1 << 20, ld_q=1 << 26, ld_qo=1 << 26) == -2
    d.head_dim = 48
    assert _apply(lib, d) == -2
    d.head_dim, d.rotary_dim = 64, 72
    assert _apply(lib, d) == -2


def test_apply_refuses_outputs_over_other_rows(lib):
    d = _rope(lib)
    row = 4 * 256
    for off in (4, -4, row, 5 * row + 4 * 255, -5 * row):
        assert _apply(lib, d, q_out=FAKE + off) == -1, off
    assert _apply(lib, d, q_out=FAKE, ld_qo=512) == -1        # another stride
    assert _apply(lib, d, q_out=FAKE, out_dtype=1) == -1      # another type
    assert _apply(lib, d, q_out=FAKE << 1) == -1              # the keys' rows
    assert _apply(lib, d, k_out=FAKE << 2) == -1              # the other output
    assert _apply(lib, d, k_out=(FAKE << 2) + 6 * row - 4) == -1


def _append(lib, rope, kv=None, layer=0, n=3, H=8, dtype=0, q=FAKE, ld_q=512, k=FAKE << 1, ld_k=256, v=FAKE << 2,
            ld_v=256, out_dtype=0, q_out=FAKE << 3, **fields):
    c = binding.KV()
    c.data, c.state, c.batch, c.capacity, c.n_layers, c.len_upper = FAKE << 4, FAKE << 4, 2, 256, 3, 200
    c.n_kv_heads, c.head_dim, c.dtype, c.window = 4, 64, binding.SPECDEC_FP8, 128
    for name, x in fields.items():
        setattr(c, name, x)
    return lib.specdec_rope_append(r(c) if kv is None else None, layer, r(rope) if rope is not None else None, n, H,
                                   dtype, q, ld_q, k, ld_k, v, ld_v, None, 0, out_dtype, q_out, None)


def test_append(lib):
    d = _rope(lib)
    for bad in ({"kv": 0}, {"layer": 3}, {"layer": -1}, {"n": 0}, {"H": 0}, {"dtype": 2}, {"out_dtype": 2}, {"q": None},
                {"k": None}, {"v": None}, {"q_out": None}, {"ld_q": 511}, {"ld_k": 255}, {"ld_v": 255}, {"data": None},
                {"state": None}, {"q_out": FAKE + 4}, {"q_out": FAKE, "ld_q": 513}, {"q_out": FAKE, "out_dtype": 1},
                {"q_out": FAKE << 1}, {"q_out": (FAKE << 2) + 4 * 256 * 6 - 4}):
        assert _append(lib, d, **bad) == -1, bad
    assert _append(lib, None) == -1
    for bad in ({"H": 6}, {"n": 66}, {"head_dim": 128}, {"head_dim": 32}):
        assert _append(lib, d, **bad) == -2, bad
    assert _append(lib, d, n=57) == -3
    plain = binding.KV()
    plain.data, plain.state, plain.batch, plain.capacity, plain.n_layers = FAKE, FAKE, 2, 256, 3
    plain.n_kv_heads, plain.head_dim, plain.dtype, plain.window = 4, 64, binding.SPECDEC_BF16, 128
    assert lib.specdec_rope_append(r(plain), 0, r(d), 1, 8, 0, FAKE, 512, FAKE << 1, 256, FAKE << 2, 256, None, 0, 0,
                                   FAKE << 3, None) == -6


def test_binding_checks():
    import torch
    with pytest.raises(ValueError):
        binding.specdec_rope_apply(None, None, None, None, None)
    with pytest.raises(ValueError):  # an output without its input
        binding.specdec_rope_apply(None, torch.zeros(1, 1, 1, 64), None, None, torch.zeros(1, 1, 1, 64))
    with pytest.raises(ValueError):
        binding._float_type(torch.float16, "x")
