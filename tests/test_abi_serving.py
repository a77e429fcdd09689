"""Host-side checks of the sampling-rule, FP8-cache and attention calls: sizes,
and the refusals that launch nothing (no GPU needed)."""
import ctypes

import pytest

from paper_2608_10362_amd import binding, synth


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(binding.LIB_PATH):
        from paper_2608_10362_amd import build
        build.build()
    return binding.lib()


FAKE = ctypes.c_void_p(4096)  # never dereferenced: the calls below fail first
ODD = ctypes.c_void_p(4100)


def test_cache_sizes_and_init_errors(lib):
    d = binding.make_desc(synth.LLAMA_7B)
    size = lambda *a: lib.specdec_kv_bytes_fp8(ctypes.byref(d), *a)  # noqa: E731
    L, B, cap, win = 32, 2, 2048, 128
    codes, ring = L * B * 32 * 2 * cap * 128, L * B * 32 * 2 * win * 128 * 2
    scales = L * B * 32 * 2 * (cap // 64) * 4
    counters = B * 32 * 4 * win * 4
    assert size(L, B, cap, win) == codes + ring + scales + counters
    assert size(L, B, cap, win) < 0.57 * lib.specdec_kv_bytes(ctypes.byref(d), L, B, cap)
    for bad in ((0, B, cap, win), (33, B, cap, win), (L, 0, cap, win), (L, B, 100, win), (L, B, cap, 64),
                (L, B, cap, 100), (L, B, -64, win)):
        assert size(*bad) == 0
    f32 = binding.make_desc(synth.TINY)
    assert lib.specdec_kv_bytes_fp8(ctypes.byref(f32), 1, 1, 64, 128) == 0
    kv = binding.KV()
    init = lambda k, desc, *a: lib.specdec_kv_init_fp8(k, desc, *a)  # noqa: E731
    kr, dr, n = ctypes.byref(kv), ctypes.byref(d), size(L, B, cap, win)
    assert init(None, dr, L, B, cap, win, FAKE, n, FAKE, None) == -1
    assert init(kr, None, L, B, cap, win, FAKE, n, FAKE, None) == -1
    assert init(kr, dr, L, B, cap, win, None, n, FAKE, None) == -1
    assert init(kr, dr, L, B, cap, win, ctypes.c_void_p(4096 + 64), n, FAKE, None) == -1
    assert init(kr, dr, L, B, cap, win, FAKE, n, ODD, None) == -1
    assert init(kr, dr, L, B, cap, win, FAKE, n - 1, FAKE, None) == -1
    assert init(kr, dr, L, B, cap, 64, FAKE, n, FAKE, None) == -2
    assert init(kr, dr, L, B, 2000, win, FAKE, n, FAKE, None) == -2
    assert init(kr, ctypes.byref(f32), 1, 1, 64, 128, FAKE, n, FAKE, None) == -6


def _cache(dtype=binding.SPECDEC_FP8, cap=256, window=128):
    kv = binding.KV()
    kv.data, kv.state, kv.batch, kv.capacity, kv.n_layers = 4096, 4096, 2, cap, 3
    kv.n_kv_heads, kv.head_dim, kv.dtype, kv.len_upper, kv.window = 4, 64, dtype, 200, window
    return kv


def test_cache_call_errors(lib):
    kv, plain = _cache(), _cache(binding.SPECDEC_BF16)
    r = ctypes.byref
    assert lib.specdec_kv_write_context(r(kv), 0, 0, 32, 10, FAKE, FAKE, None) == -2
    assert lib.specdec_kv_write_context(r(kv), 0, 0, 192, 65, FAKE, FAKE, None) == -3
    assert lib.specdec_kv_write_context(r(kv), 0, 0, 64, 2 ** 31 - 1, FAKE, FAKE, None) == -3
    assert lib.specdec_kv_read_context(r(kv), 0, 0, 250, 7, FAKE, FAKE, None) == -3
    assert lib.specdec_kv_read_context(r(kv), 3, 0, 0, 7, FAKE, FAKE, None) == -1
    assert lib.specdec_kv_append(r(plain), 0, 1, FAKE, FAKE, None) == -6
    assert lib.specdec_kv_append(r(kv), 3, 1, FAKE, FAKE, None) == -1
    assert lib.specdec_kv_append(r(kv), 0, 0, FAKE, FAKE, None) == -1
    assert lib.specdec_kv_append(r(kv), 0, 1, None, FAKE, None) == -1
    assert lib.specdec_kv_append(r(kv), 0, 66, FAKE, FAKE, None) == -2
    assert lib.specdec_kv_append(r(kv), 0, 57, FAKE, FAKE, None) == -3
    assert lib.specdec_kv_advance(r(plain), 1, None) == -6
    assert lib.specdec_kv_advance(r(kv), 0, None) == -1
    assert lib.specdec_kv_advance(r(kv), 66, None) == -2
    assert lib.specdec_kv_advance(r(kv), 57, None) == -3
    assert lib.specdec_kv_commit(r(kv), 65, 0, FAKE, FAKE, 65, FAKE, None) == -2


def test_attention_errors(lib):
    kv, plain, r = _cache(), _cache(binding.SPECDEC_BF16), ctypes.byref
    ws = lib.specdec_attention_workspace_bytes(r(kv), 8, 2)
    assert ws > 0 and ws % 256 == 0
    for bad in ((plain, 8, 2), (kv, 6, 2), (kv, 8, 0), (kv, 8, 66), (kv, 0, 1)):
        assert lib.specdec_attention_workspace_bytes(r(bad[0]), *bad[1:]) == 0
    call = lambda k, layer, H, n, q, o, w, nb: lib.specdec_attention(r(k), layer, H, n, q, o, w, nb, None)  # noqa: E731
    assert call(plain, 0, 8, 2, FAKE, FAKE, FAKE, ws) == -6
    assert call(kv, 0, 6, 2, FAKE, FAKE, FAKE, ws) == -2
    assert call(kv, 0, 8, 66, FAKE, FAKE, FAKE, 1 << 40) == -2
    assert call(kv, 0, 8, 57, FAKE, FAKE, FAKE, 1 << 40) == -3
    assert call(kv, 3, 8, 2, FAKE, FAKE, FAKE, ws) == -1
    assert call(kv, 0, 8, 2, None, FAKE, FAKE, ws) == -1
    assert call(kv, 0, 8, 2, FAKE, FAKE, FAKE, ws - 1) == -1
    assert call(kv, 0, 8, 2, FAKE, FAKE, ODD, ws) == -1


def test_sample_logits_errors(lib):
    need = lib.specdec_sample_logits_workspace_bytes
    ws = need(2, 3, 1000)
    assert ws > 0 and ws % 256 == 0
    for bad in ((0, 1, 10), (1, 0, 10), (1, 1, 0), (1, 1, 2 ** 20 + 1), (65536, 1, 10), (2 ** 20, 2 ** 12, 10)):
        assert need(*bad) == 0

    def call(batch=2, rows=3, vocab=1000, logits=4096, ld=1000, rules=None, step_dev=None, purpose=2, index=0,
             probs=1 << 30, ld_probs=1000, out=2 << 30, ld_out=1, work=4096, nbytes=ws):
        return lib.specdec_sample_logits(batch, rows, vocab, logits, ld, rules, None, 0, 0, step_dev, purpose, index,
                                         probs, ld_probs, out, ld_out, None, work, nbytes, None)

    assert call(vocab=2 ** 20 + 1, ld=2 ** 21) == -6
    for bad in ({"batch": 0}, {"logits": None}, {"ld": 999}, {"probs": None, "out": None}, {"ld_probs": 999},
                {"ld_out": 0}, {"step_dev": 4100}, {"purpose": 0x10000}, {"index": -1}, {"index": 0xfffe},
                {"work": None}, {"work": 4100}, {"nbytes": ws - 1}, {"probs": 4096}, {"probs": 4096 + 4 * 5999}):
        assert call(**bad) == -1, bad
