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
