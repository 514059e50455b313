"""The numbering of the 8-bit attention's query blocks, on the host by the device's own arithmetic."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def quant_blocks(tmp_path_factory):
    """Runs the host build of the numbering (quant_blocks_host.cpp)."""
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "no C++ compiler"
    exe = str(tmp_path_factory.mktemp("quant_blocks") / "quant_blocks_host")
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2509_16686_amd", "csrc"),
                    os.path.join(ROOT, "tests", "quant_blocks_host.cpp"), "-o", exe], check=True)

    def run(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True)
        assert r.returncode == 0, (args, r.stdout, r.stderr)
        return tuple(map(int, r.stdout.split()))
    return run


# the largest calls by tokens, heads and sequences (2^23 work-groups of 16 tokens and a head; batch 4096), and small ones
@pytest.mark.parametrize("tokens,heads,rows,batch", [(1 << 19, 256, 16, 4096), (1 << 19, 256, 128, 4096), (1 << 17, 1024, 16, 4095),
                                                     (1 << 18, 130, 16, 4000), (40, 5, 16, 3), (40, 128, 128, 3), (0, 1, 16, 1)])
def test_offsets_that_rise_and_fall_stay_in_the_numbering(quant_blocks, tokens, heads, rows, batch):
    """Every sequence's first block lies behind the one before it and within the room for blocks."""
    last, falls, outside = quant_blocks(tokens, heads, rows, batch)
    assert falls == outside == 0 and last <= tokens * heads // rows + batch
