"""Stores that fill a key tile of the 8-bit cache's attention, on the host by the device's own arithmetic."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def key_tile(tmp_path_factory):
    """Runs the host build of the stores (key_tile_host.cpp)."""
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "no C++ compiler"
    exe = str(tmp_path_factory.mktemp("key_tile") / "key_tile_host")
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2509_16686_amd", "csrc"), os.path.join(ROOT, "tests", "key_tile_host.cpp"),
                    "-o", exe], check=True)

    def run(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True)
        assert r.returncode == 0, (args, r.stdout, r.stderr)
        return tuple(map(int, r.stdout.split()))
    return run


@pytest.mark.parametrize("dc", [64, 128, 320, 512])
def test_a_tile_is_filled_without_touching_the_one_attended_to(key_tile, dc):
    """While one buffer is filled the other is read: no store reaches it, and each piece of the tile is stored once."""
    assert key_tile(dc) == (0, 0)
