"""Strides between rows that no memory holds: an error, in norm and rotation and wherever rows' overlap is looked at
(no GPU needed)."""
import subprocess
import sys

import pytest

from tests.test_rope_inputs_refusals import _append, _apply, _rope
from tests.test_rope_refusals import lib  # noqa: F401


def test_strides_that_no_memory_holds(lib):  # noqa: F811
    d = _rope(lib)
    for ld in (1 << 62, (1 << 63) - 1, 1 << 61, 1 << 56):
        for name in ("ld_q", "ld_k", "ld_qo", "ld_ko"):
            assert _apply(lib, d, **{name: ld}) == -1, (name, ld)
        for name in ("ld_q", "ld_k", "ld_v"):
            assert _append(lib, d, **{name: ld}) == -1, (name, ld)


@pytest.mark.parametrize("call", [
    "d = b.RopeDesc(); l.specdec_rope_init(r(d), 64, 64, 1e4, 0, None, None, 0, 0.0); "
    "print(l.specdec_rope_apply(r(d), 1, 1, 4, 0, 0, 1 << 20, 1 << 62, None, 0, None, 0, 0, (1 << 20) + 64, 1 << 62, None, 0, None))",
    "s = b.Sampling(); print(l.specdec_sample_logits(1, 1, 1000, 1 << 20, 1 << 62, r(s), None, 1, 1, None, 0, 0, "
    "(1 << 20) + 64, 1 << 62, None, 0, None, 1 << 20, 1 << 50, None))"], ids=["rope", "sample_logits"])
def test_a_stride_whose_bytes_wrap_to_nothing(call):
    """An error, not a division by it (which ends the process)."""
    code = f"import ctypes; from paper_2608_10362_amd import binding as b; l, r = b.lib(), ctypes.byref; {call}"
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and out.stdout.strip() == "-1", (out.returncode, out.stdout, out.stderr[-500:])
