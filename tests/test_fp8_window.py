"""The default window of an 8-bit cache (no GPU needed)."""
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


@pytest.mark.parametrize("shape", [synth.LLAMA_7B, synth.LLAMA_1B], ids=["7b", "1b"])
@pytest.mark.parametrize("rows", [1, 16, 64, 300, 2048, 8192])
@pytest.mark.parametrize("batch", [1, 3, 16])
def test_an_8_bit_cache_is_the_smaller_one_whatever_the_handles_rows(lib, shape, rows, batch):
    """Codes and scales are 0.51 of a bf16 cache, the default ring at most a quarter of one."""
    d = binding.make_desc(shape)
    for capacity in (512, 1024, 2048, 4096, 32768):
        w = binding.default_window(rows, batch, capacity)
        assert w % 64 == 0 and 128 <= w <= max(128, capacity // 4)
        n8 = lib.specdec_kv_bytes_fp8(ctypes.byref(d), 2, batch, capacity, w)
        n16 = lib.specdec_kv_bytes(ctypes.byref(d), 2, batch, capacity)
        assert 0 < n8 <= 0.80 * n16, (capacity, w, n8 / n16)


def test_the_default_takes_the_handles_rows_where_a_quarter_holds_them():
    assert binding.default_window(64, 2, 512) == 128       # 32 rows a sequence
    assert binding.default_window(300, 1, 4096) == 384     # 300 rows and the block before them
    assert binding.default_window(2048, 4, 8192) == 320     # 1024 rows a pass, 256 a sequence
    assert binding.default_window(2048, 1, 2048) == 512    # a quarter of the capacity
    assert binding.default_window(2048, 1, 32768) == 1088  # more than 1024 rows a pass bring nothing
    assert binding.default_window(0, 1, 64) == 128


@pytest.mark.parametrize("batch,capacity", [(0, 512), (-1, 512), (2, 0), (2, -64), (2, 100), (65536, 64)])
def test_sizes_without_a_cache_are_refused_as_shapes(lib, batch, capacity):
    with pytest.raises(binding.SpecdecError) as e:
        binding.Fp8KVCache(synth.LLAMA_1B, batch, capacity, n_layers=1, device="cpu")
    assert e.value.status == -2
