"""Refusals of the norm and rotation calls: outputs over positions or gains (no GPU needed)."""
import ctypes

from paper_2608_10362_amd import binding
from tests.test_rope_refusals import FAKE, lib  # noqa: F401

r = ctypes.byref
POS, GAIN, Q, K, V, OUT = (FAKE * i for i in (20, 24, 28, 32, 36, 40))


def _rope(lib, q_gain=None, k_gain=None, hd=64):
    d = binding.RopeDesc()
    assert lib.specdec_rope_init(r(d), hd, hd, 10000.0, 0, q_gain, k_gain, 0, 1e-5) == 0
    return d


def _apply(lib, d, pos=None, batch=2, n=3, ld_q=256, ld_k=128, ld_qo=256, ld_ko=128, q_out=OUT, k_out=OUT + FAKE, q=Q, k=K):
    return lib.specdec_rope_apply(r(d), batch, n, 4, 2, 0, q, ld_q, k, ld_k, pos, 0, 0, q_out, ld_qo, k_out, ld_ko, None)


def _append(lib, d, pos=None, q_out=OUT, ld_q=512, ld_k=256, ld_v=256):
    c = binding.KV()
    c.data, c.state, c.batch, c.capacity, c.n_layers, c.len_upper = FAKE, FAKE, 2, 256, 3, 200
    c.n_kv_heads, c.head_dim, c.dtype, c.window = 4, 64, binding.SPECDEC_FP8, 128
    return lib.specdec_rope_append(r(c), 0, r(d), 3, 8, 0, Q, ld_q, K, ld_k, V, ld_v, pos, 0, 0, q_out, None)


def test_an_output_over_positions(lib):  # noqa: F811
    d = _rope(lib)
    rows, row = 6, 4 * 256
    for at in (0, 4, row - 4, 5 * row, 6 * row - 4):  # (where the positions lie in the output's rows)
        assert _apply(lib, d, pos=OUT + at) == -1, at
        assert _apply(lib, d, pos=OUT + FAKE + at // 2) == -1, at
    assert _apply(lib, d, pos=OUT - 4 * rows + 4) == -1
    # rows with a gap: positions that reach into the next row
    assert _apply(lib, d, pos=OUT + 4 * (256 + 3), ld_qo=256 + 8) == -1
    assert _append(lib, d, pos=OUT) == -1 and _append(lib, d, pos=OUT + 6 * 4 * 512 - 4) == -1


def test_an_output_over_gains(lib):  # noqa: F811
    for q_gain, k_gain in ((GAIN, None), (None, GAIN)):
        d = _rope(lib, q_gain, k_gain)
        for at in (GAIN, GAIN + 4, GAIN + 4 * 63, GAIN - 4):
            assert _apply(lib, d, q_out=at) == -1 and _apply(lib, d, k_out=at) == -1
            assert _append(lib, d, q_out=at) == -1
