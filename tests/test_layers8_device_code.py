"""What the compiled kernels of the 8-bit layers have to hold and no run can show.  No GPU: the device code is compiled to assembly here."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2307_16273_amd import build


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="hipcc is not installed")
def test_tiles_wait_for_their_reads_before_the_barrier(tmp_path):
    """Behind the barrier of a stage other waves' loads write over the LDS of the stage before: in front of the
    barrier stands a wait that leaves no LDS read of this wave under way."""
    out = tmp_path / "k.s"
    r = subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "k_matmul8.hip"), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    kernel, reading, seen = None, True, {}
    for line in out.read_text().splitlines():
        label = re.match(r"(\.LBB\w+|_Z\d+(k_m8_\w+)):", line)
        if label:
            reading = True                      # whatever was under way where control comes from
            kernel = label.group(2) or kernel
        op = line.split(";")[0].split()
        if kernel is None or not op:
            continue
        if op[0].startswith("ds_read"):
            reading = True
        elif op[0] == "s_waitcnt" and "lgkmcnt(0)" in op[1:]:
            reading = False
        elif op[0] == "s_barrier" and kernel.startswith(("k_m8_tile", "k_m8_pair")):
            seen[kernel] = seen.get(kernel, 0) + 1
            assert not reading, kernel
    # three sizes of tiles in four layouts, and the pair in two with a tile of each gradient
    assert len(seen) == 14 and sorted(seen.values()) == [1] * 12 + [2] * 2, seen
