"""A server's decode step and the return of its pages, each captured once on a stream of its own and replayed with other
lengths, rows and tables in the same arrays: every replay gives the bits of the same calls made directly."""
import pytest
import torch

import server_oracle as S
from paper_2509_16686_amd import binding as B
from parity import say

pytestmark = pytest.mark.gpu
I32 = torch.int32
PAGE, BATCH, WIDTH, KEEP, POOL = 16, 6, 30, 7, 140


def ints(x):
    return torch.tensor(x, dtype=I32, device="cuda")


class Step:
    """Everything that a step reads and writes; `run` makes its calls."""

    def __init__(self, layer, seed=5):
        self.L = L = S.Layer(**layer, page=PAGE, pages=POOL + 8, seed=seed)
        dq, row = L.dh + L.dr, L.dc + L.dr
        self.x, self.new_ids = L.normal((BATCH, L.h * dq + row)), L.ints(211, BATCH)
        self.kw = L.normal((L.dr,), 0.1, 1.0)
        self.cached, self.new = ints([0] * BATCH), ints([1] * BATCH)
        self.base, self.prefix_len, self.prefix_table = ints([90] * BATCH), ints([90]), ints(list(range(POOL, POOL + 6)))
        self.table = torch.full((BATCH, WIDTH), -1, dtype=I32, device="cuda")
        self.free, self.count = torch.randperm(POOL, generator=L.g).to(I32).cuda(), ints([POOL])
        new = lambda *s, t=I32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        self.lens, self.cu, self.count_out = new(BATCH), new(BATCH + 1), new(1)
        self.positions, self.slots, self.q = new(BATCH), new(BATCH), new(BATCH, L.h, dq, t=L.dtype)
        self.means = new(POOL + 8, row, t=L.dtype)
        self.scores, self.sel = new(BATCH, WIDTH, t=torch.float32), new(BATCH, KEEP)
        self.sel_lens, self.sel_index = new(BATCH), new(BATCH, KEEP)
        self.shared, self.sparse = (new(BATCH, L.h, L.dv, t=L.dtype) for _ in range(2))
        self.ws = B.alloc_workspace(max(B.decode_shared_workspace_size(L.dims, BATCH, WIDTH, 6),
                                        B.decode_workspace_size(L.dims, BATCH, max(WIDTH, KEEP)),
                                        B.page_scores_workspace_size(L.dims, BATCH)))

    def run(self):
        L, n = self.L, self.L.h * (self.L.dh + self.L.dr)
        B.page_plan(PAGE, self.cached, self.new, self.table, self.free, self.count, self.lens, self.cu, self.positions,
                    self.slots, self.count_out, position_base=self.base)
        B.qk_norm_rope(L.dims, self.x[:, :n], self.q, self.x[:, n:], L.cache, L.ids, self.new_ids, self.positions, self.slots,
                       k_norm_w=self.kw)
        B.page_means(L.dims, L.cache, L.ids, L.gate, self.cached, self.lens, self.table, WIDTH, self.means)
        B.decode_shared(L.dims, self.q, L.cache, L.ids, L.gate, L.w_uk, L.w_uv, self.prefix_len, self.prefix_table, self.lens,
                        self.table, WIDTH, self.ws, self.shared)
        B.page_scores(L.dims, self.q, L.w_uk, self.means, self.lens, self.table, WIDTH, self.ws, self.scores)
        B.select_pages(L.dims, self.scores, self.lens, self.table, WIDTH, self.sel, self.sel_lens, keep_last=2,
                       sel_index=self.sel_index)
        B.decode(L.dims, self.q, L.cache, L.ids, L.gate, L.w_uk, L.w_uv, self.sel_lens, self.sel, KEEP, self.ws, self.sparse)

    def results(self):
        return dict(lens=self.lens, cu=self.cu, count=self.count_out, positions=self.positions, slots=self.slots, q=self.q,
                    table=self.table, cache=self.L.cache, ids=self.L.ids, means=self.means, scores=self.scores, sel=self.sel,
                    sel_lens=self.sel_lens, sel_index=self.sel_index, shared=self.shared, sparse=self.sparse)

    def advance(self, lengths, seed):
        """Other requests in the same arrays: rows of `lengths` cached tokens, fresh projections, a shorter prefix."""
        L = self.L
        L.g.manual_seed(seed)
        self.x.copy_(L.normal(tuple(self.x.shape)))
        self.cached.copy_(ints(lengths))
        self.new.copy_(ints([1, 1, 0, 1, 1, 1]))
        self.prefix_len.fill_(90 - seed)
        table, at = torch.full((BATCH, WIDTH), -1, dtype=I32), 0
        order = torch.randperm(POOL, generator=L.g).to(I32)
        for b, n in enumerate(lengths):
            k = S.ceil_div(n, PAGE)
            table[b, :k] = order[at:at + k]
            at += k
        self.table.copy_(table.cuda())
        self.free[: POOL - at] = order[at:].cuda()
        self.count.fill_(POOL - at)
        self.means.copy_(L.normal(tuple(self.means.shape), 0.3))


@pytest.mark.parametrize("layer", [dict(h=16, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),
                                   dict(h=128, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),
                                   dict(h=8, dh=64, dv=64, dc=128, dr=32, dtype="fp32")])
def test_a_captured_step_gives_the_bits_of_the_calls(gpu, layer):
    a, b = Step(layer), Step(layer)
    b.advance([16, 0, 3, 200, 31, 47], 1)
    b.run()  # module loading, before the capture
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        a.run()
    for seed, lengths in enumerate([[1, 0, 5, 17, 320, 48], [200, 16, 0, 0, 15, 479], [0] * 6], start=2):
        say(f"captured step {lengths}")
        for step in (a, b):
            step.L.cache.copy_(b.L.cache), step.L.ids.copy_(b.L.ids)
            step.advance(lengths, seed)
        g.replay()
        torch.cuda.synchronize()
        b.run()
        torch.cuda.synchronize()
        want = b.results()
        for name, got in a.results().items():
            assert torch.equal(got, want[name]), name
        assert bool(torch.isfinite(a.shared.float()).all()) and bool(torch.isfinite(a.sparse.float()).all())


def test_a_captured_release_replays(gpu):
    say("page_release captured")
    rows, free, lens, ended = ints([0] * 40).reshape(8, 5), torch.full((64,), -1, dtype=I32, device="cuda"), ints([0] * 8), ints([0] * 8)
    count, out, count_out = ints([0]), ints([0] * 8), ints([0])
    B.page_release(PAGE, lens, ended, rows, free, count, out, count_out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        B.page_release(PAGE, lens, ended, rows, free, count, out, count_out)
    gen = torch.Generator().manual_seed(3)
    for held in (0, 7, 50):
        table = torch.randperm(40, generator=gen).to(I32)
        n, e = torch.randint(0, 81, (8,), generator=gen).to(I32), torch.randint(0, 2, (8,), generator=gen).to(I32)
        rows.copy_(table.reshape(8, 5)), lens.copy_(n), ended.copy_(e), count.fill_(held), free.fill_(-1)
        g.replay()
        torch.cuda.synchronize()
        want = S.page_release(PAGE, n.numpy(), e.numpy(), table.reshape(8, 5).numpy(), torch.full((64,), -1).numpy(), held)
        assert free.tolist() == list(want[0]) and out.tolist() == list(want[1]) and int(count_out) == want[2]
