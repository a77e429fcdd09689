"""The wait state between M0's write and a load to LDS, in the shared prefix's attention (see test_device_asm)."""
from tests.test_device_asm import test_m0_settles_before_a_load_to_lds as check


def test_m0_settles_before_a_ring_row_goes_to_lds(tmp_path):
    check("attention_shared.hip", tmp_path)
