"""Refusals of the 8-bit cache's and the sampling calls that launch nothing (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2608_10362_amd import binding


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(binding.LIB_PATH):
        from paper_2608_10362_amd import build
        build.build()
    return binding.lib()


class _Cache:
    """As much of an Fp8KVCache as a call's argument checks see."""
    def __init__(self, device):
        self.data = torch.zeros(1, dtype=torch.uint8, device=device)
        self.kv = binding.KV()


def test_an_advance_takes_a_cache_on_the_current_device(monkeypatch):
    called = []
    monkeypatch.setattr(binding, "lib", lambda: type("L", (), {"specdec_kv_advance": lambda *a: called.append(a) or 0}))
    monkeypatch.setattr(binding, "_stream", lambda s: None)
    with pytest.raises(ValueError):
        binding.specdec_kv_advance(_Cache("cpu"), 1)
    assert not called


FAKE = 1 << 20  # never dereferenced: the calls fail first


def _attention(lib, q, out, batch=2, n_kv_heads=4, head_dim=64, n_heads=8, n=2, window=128, capacity=256):
    kv = binding.KV()
    kv.data, kv.state, kv.batch, kv.capacity, kv.n_layers, kv.len_upper = FAKE, FAKE, batch, capacity, 3, 100
    kv.n_kv_heads, kv.head_dim, kv.dtype, kv.window = n_kv_heads, head_dim, binding.SPECDEC_FP8, window
    return lib.specdec_attention(ctypes.byref(kv), 0, n_heads, n, q, out, FAKE, 1 << 60, None)


def test_attention_refuses_an_out_that_is_part_of_q(lib):
    nbytes = 2 * 2 * 8 * 64 * 4
    for off in (4, 256, nbytes - 4):
        assert _attention(lib, FAKE, FAKE + off) == -1
        assert _attention(lib, FAKE + off, FAKE) == -1


def _desc(n_heads, n_kv_heads, head_dim=32, d_model=64):
    from paper_2608_10362_amd.synth import ModelShape
    return binding.make_desc(ModelShape(1, d_model, n_heads, n_kv_heads, head_dim, 64, 64))


def test_sizes_past_the_attentions_grid_are_shapes_not_hip_errors(lib):
    assert _attention(lib, FAKE, FAKE, batch=65536) == -2
    # 17 query tiles of 32 in each of 8192 kv heads; 8 tiles
    assert _attention(lib, FAKE, FAKE, n_kv_heads=8192, n_heads=65536, n=65) == -2
    assert _attention(lib, FAKE, FAKE, n_kv_heads=8192, n_heads=65536, n=32) == -2
    kv = binding.KV()
    kv.data, kv.state, kv.batch, kv.capacity, kv.n_layers = FAKE, FAKE, 1, 256, 1
    kv.n_kv_heads, kv.head_dim, kv.dtype, kv.window = 8192, 64, binding.SPECDEC_FP8, 128
    assert lib.specdec_attention_workspace_bytes(ctypes.byref(kv), 65536, 65) == 0
    assert lib.specdec_attention_workspace_bytes(ctypes.byref(kv), 65536, 28) > 0
    kv.batch = 65536
    assert lib.specdec_attention_workspace_bytes(ctypes.byref(kv), 8192, 1) == 0
    assert lib.specdec_kv_bytes_fp8(ctypes.byref(_desc(8, 8)), 1, 65535, 64, 128) > 0
    assert lib.specdec_kv_bytes_fp8(ctypes.byref(_desc(8, 8)), 1, 65536, 64, 128) == 0


def test_passes_past_the_attentions_grid_launch_nothing(lib):
    d = _desc(65536, 8192)
    ptrs = (ctypes.c_void_p * 1)(FAKE)
    w = binding.Weights(FAKE, FAKE, FAKE, *[ctypes.cast(ptrs, binding._PP)] * 9)
    ws = lib.specdec_workspace_bytes(ctypes.byref(d), 128, 256)
    m = ctypes.c_void_p()
    assert lib.specdec_model_create(ctypes.byref(d), ctypes.byref(w), 1, FAKE, 1 << 60, 128, 256, FAKE, ws,
                                    ctypes.byref(m)) == 0
    kv = binding.KV()
    kv.data, kv.state, kv.batch, kv.capacity, kv.n_layers, kv.window = FAKE, FAKE, 1, 256, 1, 128
    kv.n_kv_heads, kv.head_dim, kv.dtype = 8192, 32, binding.SPECDEC_FP8
    assert lib.specdec_verify(m, ctypes.byref(kv), 64, FAKE, 64, FAKE, None) == -2
    # (a prompt's chunks hold window - 64 tokens: 64, 16 tiles in each of 8192 kv heads)
    assert lib.specdec_prefill(m, ctypes.byref(kv), 80, FAKE, None) == -2
    lib.specdec_model_destroy(m)


def test_probabilities_over_the_logits_are_refused(lib):
    ws = lib.specdec_sample_logits_workspace_bytes(2, 3, 1000)

    def call(probs, ld=2000, ld_probs=2000):
        return lib.specdec_sample_logits(2, 3, 1000, FAKE, ld, None, None, 0, 0, None, 2, 0, probs, ld_probs, None, 0,
                                         None, FAKE, ws, None)
    for at in (0, 4, 3996, 4004, 8000, 8000 * 5 + 3996, -3996, -8000 * 5 - 3996):  # (a row ends at 4000, the next starts at 8000)
        assert call(FAKE + at) == -1, at
    for at in (4000, 8000, -4000):  # other strides
        assert call(FAKE + at, ld_probs=1000) == -1 and call(FAKE + at, ld=1000) == -1
