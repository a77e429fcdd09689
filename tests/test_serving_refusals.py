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
