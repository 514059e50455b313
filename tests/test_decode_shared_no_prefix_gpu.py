"""eg_mla_decode_shared without prefix pages is eg_mla_decode: the same bits."""
import pytest
import torch

from paper_2509_16686_amd import binding as B
from parity import say
from test_decode_shared_gpu import LAYERS, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layer", sorted(LAYERS))
@pytest.mark.parametrize("lens", [[1], [700, 0, 65], [(91 * b) % 400 for b in range(40)]], ids=len)
@pytest.mark.parametrize("paged", [True, False])
def test_bits_of_decode(gpu, layer, lens, paged):
    say(f"decode_shared without prefix {layer} batch={len(lens)} paged={paged}")
    c = Case(layer, 0, lens, extra_pages=len(lens) * 12)
    L, width = c.L, c.table.shape[1]
    table = c.table if paged else None
    got, want = torch.full_like(c.out, 7), torch.full_like(c.out, 9)
    n = B.decode_shared_workspace_size(L.dims, len(lens), width, 0)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    B.decode_shared(L.dims, c.q, L.cache, L.ids, L.gate, L.w_uk, L.w_uv, None, None, c.seq_lens, table, width, ws, got)
    ws = B.alloc_workspace(B.decode_workspace_size(L.dims, len(lens), width))
    B.decode(L.dims, c.q, L.cache, L.ids, L.gate, L.w_uk, L.w_uv, c.seq_lens, table, width, ws, want)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
