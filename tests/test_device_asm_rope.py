"""The assembly of the rotation's kernels into a cache: values cross the lanes of a wave through LDS, and
nothing but a barrier of the wave tells the compiler that a lane reads what others wrote.  Each group of
such stores is followed by one before the reads, and the reads by one before the next unit's stores.
No GPU needed: hipcc writes the assembly."""
import os
import re
import subprocess

from paper_2608_10362_amd import build


def _kernels(src, tmp_path):
    """name -> events of its text in order: W (16 bytes stored to LDS), R (16 loaded), B (a wave's barrier)."""
    out = str(tmp_path / (src + ".s"))
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([build.HIPCC, *flags, "--offload-device-only", "-S", "-I", build.INCLUDE, "-I", build.CSRC,
                    os.path.join(build.CSRC, src), "-o", out], check=True, stdout=subprocess.PIPE,
                   stderr=subprocess.STDOUT, timeout=600)
    kernels, events = {}, None
    for line in open(out):
        name = re.match(r"(_Z\w+):", line)
        if name:
            events = kernels[name.group(1)] = []
        elif events is not None:
            for event, at in (("W", r"\s*ds_write_b128\b"), ("R", r"\s*ds_read_b128\b"), ("B", r"\s*; wave barrier")):
                if re.match(at, line):
                    events.append(event)
    return {name: "".join(e) for name, e in kernels.items()}


def test_values_cross_lanes_behind_a_barrier(tmp_path):
    cached = {name: e for name, e in _kernels("rope.hip", tmp_path).items() if "W" in e}
    assert len(cached) == 12  # (3 head sizes, 2 x 2 types)
    for name, events in cached.items():
        # (the loop over units may start behind its last barrier or with it)
        assert re.search(r"W{8}BR{8}B|BW{8}BR{8}", events), (name, events)
        assert not re.search(r"WR|RW", events), (name, events)
