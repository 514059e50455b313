"""Captured calls of eg_mla_quant_attend: one graph for every step of a server, whose lengths, offsets and rows change between
replays, beside another graph that shares its workspace in order."""
import pytest
import torch

from paper_2509_16686_amd import binding as B
from quant_oracle import BF, I32, Layer, check_attend, ints, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(16, 128, 128, 128, 64), (16, 128, 128, 320, 64), (5, 40, 56, 48, 24)])
@pytest.mark.parametrize("width", [32, 1 << 16])  # (of 16 tokens: blocks of 16 rows; of 128 for the first two)
def test_replays_with_other_lengths(gpu, shape, width):
    L = Layer(80, *shape, page=16, rows=16 * 100)
    b, most = 3, 40
    q = L.normal((most, L.h, L.dh + L.dr))
    cu, lens = offsets([1, 1, 1]), ints([1, 1, 1])
    table = torch.zeros((b, width), dtype=I32, device="cuda")
    ws = B.alloc_workspace(B.quant_attend_workspace_size(L.dims, b, most, width)).fill_(0x5A)
    out, other = torch.empty((most, L.h, L.dv), dtype=BF, device="cuda"), torch.empty((b, L.h, L.dv), dtype=BF, device="cuda")
    step = lambda: B.quant_attend(L.dims, q, cu, L.codes, L.scales, L.w_uk, L.w_uv, lens, table, width, ws, out)
    decode = lambda: B.quant_attend(L.dims, q[:b], None, L.codes, L.scales, L.w_uk, L.w_uv, lens, table, width, ws, other)
    graphs = []
    for call in (step, decode):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for i, (new, n) in enumerate([([1, 1, 1], [5, 400, 33]), ([20, 0, 20], [20, 77, 500]), ([3, 30, 7], [100, 31, 7]), ([0, 0, 0], [9, 9, 9]),
                                  ([40, 0, 0], [512, 1, 0])]):
        cu.copy_(offsets(new))
        lens.copy_(ints(n))
        t = L.table(n)
        table.zero_()
        table[:, : t.shape[1]] = t
        q.copy_(L.normal(q.shape))
        out.fill_(7.0)
        for g in graphs if i % 2 else graphs[::-1]:
            g.replay()
        total = sum(new)
        check_attend(out[:total], *L.oracle(q[:total], new, n, L.slots_of(t))) if total else None
        assert bool((out[total:] == 7).all())
        check_attend(other, *L.oracle(q[:b], [1] * b, n, L.slots_of(t)))
        eager = torch.full_like(out, 7.0)
        B.quant_attend(L.dims, q, cu, L.codes, L.scales, L.w_uk, L.w_uv, lens, table, width, ws, eager)
        assert torch.equal(out, eager)
