"""The shared decode's plan, on the host."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def shared_plan(tmp_path_factory):
    """Runs the host build of the plan (shared_plan_host.cpp)."""
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "no C++ compiler"
    exe = str(tmp_path_factory.mktemp("shared_plan") / "shared_plan_host")
    csrc = os.path.join(ROOT, "paper_2509_16686_amd", "csrc")
    subprocess.run([cxx, "-O2", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(ROOT, "tests", "shared_plan_host.cpp"), os.path.join(csrc, "host_plan.cpp"), "-o", exe],
                   check=True)

    def run(*args):
        r = subprocess.run([exe, *map(str, args)], capture_output=True, text=True)
        assert r.returncode == 0, (args, r.stdout, r.stderr)
        return tuple(map(int, r.stdout.split()))
    return run


# heads, d_h, d_v, d_c, d_r, bf16
LAYERS = [(16, 128, 128, 128, 64, 1), (128, 128, 128, 512, 64, 1), (16, 128, 128, 320, 64, 1), (32, 128, 128, 512, 64, 1),
          (5, 128, 128, 128, 64, 1), (20, 128, 128, 320, 64, 1), (3, 128, 128, 512, 64, 1), (1, 128, 128, 128, 64, 1),
          (12, 64, 64, 64, 64, 1), (12, 64, 64, 128, 64, 1), (12, 64, 64, 256, 64, 1), (12, 64, 64, 320, 64, 1),
          (8, 64, 64, 512, 64, 1), (16, 64, 64, 128, 64, 1), (8, 64, 64, 128, 32, 0), (3, 64, 72, 400, 0, 0),
          (6, 64, 40, 32, 128, 1)]


@pytest.mark.parametrize("layer", LAYERS, ids=str)
def test_kernels_are_the_layers(shared_plan, layer):
    """Whatever the batch, both parts run on the kernels of the layer's decode, and so with its arithmetic."""
    assert shared_plan("layer", *layer) == (0,)


H128 = (128, 128, 128, 512, 64, 1)


@pytest.mark.parametrize("page,batch,pages,prefix,splits", [
    (64, 1, 64, 1, 128), (16, 8, 250, 1, 32), (64, 4, 1024, 4, 64), (32, 2, 3, 1, 3),  # few prefix tiles, many own ones
    (64, 64, 24, 125, 4), (64, 1, 1, 125, 250), (64, 300, 64, 1, 1), (32, 1, 0, 5, 5),
])
def test_splits_of_the_fused_kernel_follow_the_longer_part(shared_plan, page, batch, pages, prefix, splits):
    """Its work-groups take own tokens as well as the prefix's: as many as fill the chip while either part has tiles."""
    got = shared_plan("plan", *H128, page, batch, pages, prefix)
    assert got[3:7] == (1, 1, splits, batch)


@pytest.mark.parametrize("layer", LAYERS, ids=str)
@pytest.mark.parametrize("page,batch,pages,prefix", [(64, 300, 64, 128), (16, 128, 300, 600), (1, 40, 3000, 9000)])
def test_a_workspace_serves_smaller_calls(shared_plan, layer, page, batch, pages, prefix):
    """No smaller batch, own or prefix table asks for more than the largest, and every plan's rows end within its own."""
    assert shared_plan("sizes", *layer, page, batch, pages, prefix) == (0,)
