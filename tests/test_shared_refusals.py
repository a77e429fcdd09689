"""Refusals of the attention over a shared prefix that launch nothing (no GPU needed)."""
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


def _cache(**fields):
    kv = binding.KV()
    kv.data, kv.state, kv.batch, kv.capacity, kv.n_layers, kv.len_upper = FAKE, FAKE, 2, 256, 3, 200
    kv.n_kv_heads, kv.head_dim, kv.dtype, kv.window = 4, 64, binding.SPECDEC_FP8, 128
    for name, x in fields.items():
        setattr(kv, name, x)
    return kv


def _bytes(lib, p=None, kv=None, H=8, n=2, dtype=0):
    return lib.specdec_attention_shared_workspace_bytes(r(p or _cache()), r(kv or _cache()), H, n, dtype)


def _call(lib, p=None, kv=None, at=0, layer=0, H=8, n=2, dtype=0, q=FAKE, out=FAKE << 1, ws=FAKE, nbytes=1 << 50):
    return lib.specdec_attention_shared(r(p or _cache()), at, r(kv or _cache()), layer, H, n, dtype, q, out, ws, nbytes,
                                        None)


def test_workspace(lib):
    own = lib.specdec_attention_workspace_bytes(r(_cache()), 8, 2)
    for dtype in (0, 1):
        ws = _bytes(lib, dtype=dtype)
        assert ws > own and ws % 256 == 0
        assert _bytes(lib, p=_cache(capacity=1 << 16), dtype=dtype) > ws
    bad = [{"p": _cache(dtype=1)}, {"kv": _cache(dtype=1)}, {"p": _cache(n_kv_heads=8)}, {"p": _cache(head_dim=128)},
           {"H": 6}, {"n": 0}, {"n": 66}, {"dtype": 2}, {"p": _cache(data=None)}, {"kv": _cache(batch=65536)},
           {"kv": _cache(batch=65535, n_kv_heads=64), "p": _cache(n_kv_heads=64), "H": 64}]
    for b in bad:
        assert _bytes(lib, **b) == 0, b
    assert lib.specdec_attention_shared_workspace_bytes(None, r(_cache()), 8, 2, 0) == 0
    assert lib.specdec_attention_shared_workspace_bytes(r(_cache()), None, 8, 2, 0) == 0


def test_calls(lib):
    ws = _bytes(lib)
    for bad in ({"at": -1}, {"at": 2}, {"layer": 3}, {"layer": -1}, {"p": _cache(n_layers=1), "layer": 1}, {"q": None},
                {"out": None}, {"ws": None}, {"ws": FAKE + 4}, {"nbytes": ws - 1}, {"dtype": 2},
                {"p": _cache(state=None)}, {"n": 0}, {"H": 0}):
        assert _call(lib, **bad) == -1, bad
    for bad in ({"p": _cache(n_kv_heads=2)}, {"p": _cache(head_dim=32)}, {"H": 6}, {"n": 66}, {"H": 4 * 129},
                {"kv": _cache(batch=65536)}):
        assert _call(lib, **bad) == -2, bad
    assert _call(lib, kv=_cache(batch=65535, window=192, capacity=1024), n=17) == -2  # (rows of a kv head: 2^20 and more)
    assert _call(lib, n=57) == -3 and _call(lib, p=_cache(len_upper=257)) == -3
    assert _call(lib, p=_cache(dtype=1)) == -6 and _call(lib, kv=_cache(dtype=1)) == -6


@pytest.mark.parametrize("dtype", [0, 1])
def test_an_out_that_is_part_of_q(lib, dtype):
    nbytes = 2 * 2 * 8 * 64 * (2 if dtype else 4)
    for off in (2, 256, nbytes - 2):
        assert _call(lib, dtype=dtype, out=FAKE + off) == -1
        assert _call(lib, dtype=dtype, q=FAKE + off, out=FAKE) == -1
