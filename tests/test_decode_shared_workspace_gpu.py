"""One workspace, sized at a server's largest call, for its smaller ones: each is taken, right, and stays inside it."""
import pytest
import torch

from paper_2509_16686_amd import binding as B
from parity import assert_close, say
from test_decode_shared_gpu import Case

pytestmark = pytest.mark.gpu
GUARD = 4096


@pytest.mark.parametrize("layer", ["h16", "mla320", "h128", "h32dc512", "kv64", "h5", "rope128", "f32", "tiny", "f32wide"])
def test_smaller_calls(gpu, layer):
    say(f"decode_shared one workspace {layer}")
    dims = Case(layer, 1, [1]).L.dims
    n = B.decode_shared_workspace_size(dims, 64, 16, 32)
    ws = torch.full((n + GUARD,), 255, dtype=torch.uint8, device="cuda")
    for prefix, batch, top in [(2048, 64, 300), (2048, 31, 300), (500, 63, 90), (1000, 3, 1024), (65, 1, 1), (0, 40, 64), (300, 7, 0)]:
        c = Case(layer, prefix, [(91 * b + 1) % (top + 1) for b in range(batch)], own_width=1)
        c.check(f"{layer} prefix={prefix} batch={batch}", ws=ws[:n])
        assert_close(c.run(ws=ws[:n], pre=False), c.ref(prefix=0), c.L.storage, "no prefix pages")
        assert bool((ws[n:] == 255).all())


def test_size_of_the_largest_batch_is_enough(gpu):
    # 126 sequences of this layer asked for more than 128
    c = Case("f32", 2000, [20 + b % 40 for b in range(126)], own_width=64, extra_pages=96)
    n = B.decode_shared_workspace_size(c.L.dims, 128, 64, 128)
    ws = torch.full((n + GUARD,), 255, dtype=torch.uint8, device="cuda")
    c.check("f32 126 sequences in the workspace of 128", ws=ws[:n])
    assert bool((ws[n:] == 255).all())
