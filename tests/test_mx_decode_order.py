"""The streamed product waits for a chunk's weights, which go to LDS, through the scale
bytes that it loads behind them: in the compiled kernels no load into registers stands
between a chunk's requests, and a barrier to the compiler's scheduler stands behind them."""
import os
import re
import subprocess

import pytest

from paper_2411_17525_amd import build as B


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{name: lines} of the assembly of mx_decode.hip, built with the library's flags."""
    out = str(tmp_path_factory.mktemp("asm") / "mx_decode.s")
    flags = [f for f in B.COMMON if f != "-fPIC"]
    cmd = [B.hipcc(), *flags, "-w", "-x", "hip", "--offload-device-only", "-S",
           os.path.join(B.CSRC, "mx_decode.hip"), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True)
    found, name = {}, None
    with open(out) as f:
        for line in f:
            start = re.match(r"(_Z\w*mx_decode\w*):", line)
            if start:
                name = start[1]
                found[name] = []
            elif name:
                found[name].append(line.strip())
                if line.strip().startswith("s_endpgm"):
                    name = None
    return found


def test_every_kernel_is_there(kernels):
    # two formats: without a rotation and with five group sizes inside, one and two row tiles
    assert len(kernels) == 2 * (6 + 2)


def test_scales_are_loaded_behind_their_weights(kernels):
    for name, lines in kernels.items():
        # to LDS "L", into registers "G", the scheduler's barrier "|", branches and labels "."
        marks = ""
        for line in lines:
            if line.startswith("buffer_load") and line.endswith(" lds"):
                marks += "L"
            elif line.startswith(("global_load", "buffer_load", "flat_load")):
                marks += "G"
            elif "sched_barrier mask(0x00000000)" in line:
                marks += "|"
            elif line.startswith(("s_cbranch", "s_branch", ".LBB")):
                marks += "."
        requests = re.findall(r"L[^L]*L[^L]*L[^L]*L", marks)
        # the first chunk's and both unrolled steps'
        assert len(requests) == 3 and marks.count("L") == 12, (name, marks)
        assert all(r == "LLLL" for r in requests), (name, requests)
        assert len(re.findall(r"LLLL\|", marks)) == 3, (name, marks)
