"""Direct loads in the generated gfx950 code of the sources that have compiler flags of their own (no GPU)."""
import os
import shutil
import subprocess

import pytest

from paper_2402_19481_amd import build


def _compile(flags, source, out):
    subprocess.run(["hipcc", *flags, "--offload-device-only", "-S", os.path.join(build.CSRC, source), "-o", str(out)], check=True, capture_output=True)
    return out.read_text()


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs the compiler")
@pytest.mark.parametrize("source", sorted(build.SOURCE_FLAGS))
def test_every_direct_load_follows_its_own_write_of_m0(source, tmp_path):
    """A direct load takes its LDS address from M0: the last write of it before a load must be of the load's own kind, the
    instructions' or the compiler's.  With the flags that the library's code is compiled with."""
    inside, last, loads = False, None, 0
    for line in _compile(build.flags(source), source, tmp_path / "k.s").splitlines():
        if line.startswith("_Z"):
            last = None
        if "#ASMSTART" in line or "#ASMEND" in line:
            inside = "#ASMSTART" in line
        op = line.split(";")[0].split()
        if len(op) > 1 and op[0].startswith("s_") and op[1] == "m0,":
            last = inside
        if op and (op[0].startswith("global_load_lds") or (op[0].startswith("buffer_load") and op[-1] == "lds")):
            loads += 1
            assert last is inside, (loads, line)
    assert loads > 0


def test_flags_of_a_source():
    assert build.flags("api.hip") == build.FLAGS
    for source, own in build.SOURCE_FLAGS.items():
        assert source in build.SOURCES and build.flags(source) == build.FLAGS + own
