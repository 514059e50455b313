"""eg_mla_page_means, eg_mla_page_scores and eg_mla_select_pages against their formulas in 64 bits.

Means are rounded once: half a step of the storage type (the sum's own error, in 64 bits, is far below it).  Scores are
fp32: a sum of n products formed in any order is off by at most n 2^-24 times the sum of the products' sizes; the
absorbed query is such a sum of d_h products, the score one of d_c + d_r, and what the query's parts leave out is below
2^-24 of it.  The selection is exact."""
import numpy as np
import pytest
import torch

import server_oracle as S
from paper_2509_16686_amd import binding as B
from parity import assert_close, say

pytestmark = pytest.mark.gpu
I32 = torch.int32
LAYERS = {
    "h16": dict(h=16, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),
    "kv64": dict(h=12, dh=64, dv=64, dc=64, dr=64, dtype="bf16"),
    "mla320": dict(h=16, dh=128, dv=128, dc=320, dr=64, dtype="bf16"),
    "h128": dict(h=128, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),
    "odd": dict(h=5, dh=24, dv=8, dc=40, dr=8, dtype="bf16"),
    "h37": dict(h=37, dh=64, dv=64, dc=72, dr=0, dtype="bf16"),
    "top": dict(h=17, dh=64, dv=64, dc=576, dr=64, dtype="bf16"),
    "tiny": dict(h=4, dh=32, dv=32, dc=32, dr=0, dtype="fp32"),
    "f32": dict(h=8, dh=64, dv=64, dc=128, dr=32, dtype="fp32"),
    "f32top": dict(h=3, dh=64, dv=64, dc=604, dr=36, dtype="fp32"),
}


def cuda_ints(x):
    return torch.tensor(x, dtype=I32, device="cuda")


class Cache:
    def __init__(self, layer, lens, page=16, seed=2, width=None):
        self.lens, self.page = list(lens), page
        self.L = S.Layer(**LAYERS[layer], page=page, pages=sum(S.ceil_div(max(n, 0), page) for n in lens) + 2, seed=seed)
        self.table, _ = self.L.table([max(n, 0) for n in lens], width)
        self.width = self.table.shape[1]
        self.seq_lens = cuda_ints(lens)
        self.means = self.L.normal((self.L.pages, self.L.dc + self.L.dr), 0.3)

    def mean_refs(self, first=None):
        """(page, mean) of every page that a call with these first tokens changes."""
        t, out = self.table.cpu().numpy(), []
        for b, n in enumerate(self.lens):
            f = 0 if first is None else max(first[b], 0)
            for p in range(f // self.page, S.ceil_div(max(n, 0), self.page)):
                if f < n:
                    out.append((t[b, p], self.L.rows([t[b, p]], min(self.page, n - p * self.page)).mean(0)))
        return out

    def check_means(self, first=None):
        before = self.L.f64(self.means)
        B.page_means(self.L.dims, self.L.cache, self.L.ids, self.L.gate, None if first is None else cuda_ints(first),
                     self.seq_lens, self.table, self.width, self.means)
        torch.cuda.synchronize()
        after, half = self.L.f64(self.means), 2.0 ** -8 if self.L.storage == "bf16" else 2.0 ** -24
        changed = set()
        for p, ref in self.mean_refs(first):
            changed.add(p)
            assert np.all(np.abs(after[p] - ref) <= half * (1 + 2.0 ** -20) * np.abs(ref) + 1e-38), p
        for p in set(range(self.L.pages)) - changed:
            assert np.array_equal(after[p], before[p]), p  # left as they were

    def scores(self, q, ws=None, stream=None, table=True):
        out = torch.full((len(self.lens), self.width), 7.0, device="cuda")
        if ws is None:
            ws = torch.full((B.page_scores_workspace_size(self.L.dims, len(self.lens)),), 255, dtype=torch.uint8, device="cuda")
        B.page_scores(self.L.dims, q, self.L.w_uk, self.means, self.seq_lens, self.table if table else None, self.width, ws,
                      out, stream=stream)
        torch.cuda.synchronize()
        return out

    def check_scores(self, q):
        L, got = self.L, self.scores(q).double().cpu().numpy()
        q64, w, m, t = L.f64(q), L.f64(L.w_uk), L.f64(self.means), self.table.cpu().numpy()
        qf = L.absorbed(q64)
        size = np.einsum("bhd,hdc->bhc", np.abs(q64[..., : L.dh]), np.abs(w))  # sum of the products' sizes
        worst = 0.0
        for b, n in enumerate(self.lens):
            k = S.ceil_div(max(n, 0), self.page)
            assert np.all(got[b, k:] == -np.inf)
            if k:
                rows = m[t[b, :k]]
                ref = (L.tau * qf[b] @ rows.T).max(0)
                off = L.tau * ((L.dh + 1) * size[b] @ np.abs(rows[:, : L.dc]).T
                               + (L.dc + L.dr + 4) * np.abs(qf[b]) @ np.abs(rows).T).max(0) * 2.0 ** -24 + 1e-37
                worst = max(worst, float(np.max(np.abs(got[b, :k] - ref) / off)))
        say(f"  scores worst err/bound={worst:.3f}")
        assert worst <= 1.0


@pytest.mark.parametrize("layer", sorted(LAYERS))
@pytest.mark.parametrize("page", [1, 16, 24, 64])
def test_means_and_scores(gpu, layer, page):
    say(f"page means and scores {layer} page={page}")
    c = Cache(layer, [1, 0, 15, 16, 17, 100, 333, -3, 5 * page], page)
    c.check_means()
    c.check_scores(c.L.query(9))


@pytest.mark.parametrize("layer", ["h16", "h128", "f32"])
def test_means_of_a_step(gpu, layer):
    say(f"page means of a step {layer}")
    c = Cache(layer, [100, 64, 65, 1, 0, 200], 16)
    c.check_means(first=[99, 63, 64, 0, 0, 150])   # one token, a page's last, a page's first, the first, none, many
    c.check_means(first=[100, 90, -7, 1, 5, 2 ** 31 - 1])  # nothing new, past the end, below zero


def test_means_do_not_depend_on_when_they_are_formed(gpu):
    say("page means twice")
    c = Cache("h16", [700, 33], 64)
    c.check_means()
    once = c.means.clone()
    c.check_means(first=[640, 0])
    assert torch.equal(once, c.means)


def test_means_skip_pages_outside_the_cache(gpu):
    say("page means bad pages")
    c = Cache("h16", [48, 20], 16)
    c.table[0, 1], c.table[1, 0] = -9, 2 ** 31 - 1
    c.L.ids[::5], c.L.ids[1::5] = -4, 2 ** 31 - 1
    before = c.means.clone()
    B.page_means(c.L.dims, c.L.cache, c.L.ids, c.L.gate, None, c.seq_lens, c.table, c.width, c.means)
    torch.cuda.synchronize()
    good = {int(p) for p in (c.table[0, 0], c.table[0, 2], c.table[1, 1])}
    for p in range(c.L.pages):
        assert p in good or torch.equal(c.means[p], before[p])
    assert bool(torch.isfinite(c.scores(c.L.query(2))[:, :2]).all())  # read from clamped pages


@pytest.mark.parametrize("layer,batch,top", [("h16", 3, 40000), ("h128", 2, 9000), ("kv64", 33, 1500), ("f32", 5, 6000)])
def test_long_contexts(gpu, layer, batch, top):
    say(f"page scores {layer} batch={batch} top={top}")
    c = Cache(layer, [top - 997 * b % top for b in range(batch)], 64)
    c.check_means()
    c.check_scores(c.L.query(batch, 3.0))


def test_contiguous_pages(gpu):
    say("page means and scores without a table")
    c = Cache("h16", [30, 48, 7], 16, width=3)
    c.L = S.Layer(**LAYERS["h16"], page=16, pages=9, seed=4)
    c.table = torch.arange(9, dtype=I32, device="cuda").reshape(3, 3)
    c.means = c.L.normal((9, 192), 0.3)
    with_table = c.means.clone()
    B.page_means(c.L.dims, c.L.cache, c.L.ids, c.L.gate, None, c.seq_lens, c.table, 3, with_table)
    B.page_means(c.L.dims, c.L.cache, c.L.ids, c.L.gate, None, c.seq_lens, None, 3, c.means)
    torch.cuda.synchronize()
    assert torch.equal(with_table, c.means)
    q = c.L.query(3)
    assert torch.equal(c.scores(q), c.scores(q, table=False))
    sel = [torch.empty(3, 2, dtype=I32, device="cuda") for _ in range(2)]
    n = torch.empty(3, dtype=I32, device="cuda")
    scores = c.scores(q)
    for out, table in zip(sel, (c.table, None)):
        B.select_pages(c.L.dims, scores, c.seq_lens, table, 3, out, n)
    torch.cuda.synchronize()
    assert torch.equal(*sel)


def run_select(scores, lens, page, keep, first, last, table=None):
    b, width = scores.shape
    dims = B.make_dims(num_heads=16, head_dim=128, v_head_dim=128, latent_dim=128, rope_dim=64, vocab_size=9, page_size=page)
    if table is None:
        table = torch.randint(0, 10 ** 6, (b, width), dtype=I32, generator=torch.Generator().manual_seed(b)).cuda()
    sel, index = (torch.full((b, keep), -7, dtype=I32, device="cuda") for _ in range(2))
    n = torch.full((b,), -7, dtype=I32, device="cuda")
    B.select_pages(dims, scores, cuda_ints(lens), table, width, sel, n, keep_first=first, keep_last=last, sel_index=index)
    torch.cuda.synchronize()
    cols, tokens = S.select(scores.cpu().numpy(), np.clip(lens, 0, width * page), page, keep, first, last)
    t = table.cpu().numpy()
    for i, c in enumerate(cols):
        pad = [-1] * (keep - len(c))
        assert index[i].tolist() == c + pad, (i, lens[i])
        assert sel[i].tolist() == [int(t[i, j]) for j in c] + pad
    assert n.tolist() == tokens


@pytest.mark.parametrize("width,keep", [(1, 1), (5, 3), (64, 7), (257, 64), (1024, 64), (1025, 3), (2500, 300), (9000, 1000),
                                        (70, 100)])
@pytest.mark.parametrize("kind", ["normal", "few", "equal"])
def test_selection(gpu, width, keep, kind):
    say(f"select_pages width={width} keep={keep} {kind}")
    g = torch.Generator().manual_seed(width + keep)
    page, b = 16, 7
    scores = torch.randn((b, width), generator=g)
    if kind == "few":  # many equal scores
        scores = (scores * 2).round() / 2
    if kind == "equal":
        scores.fill_(-0.25)
    lens = [width * page, 0, 1, max(1, width * page // 2), min(width * page, keep * page + 1), width * page - 5, 2 ** 31 - 1]
    for first, last in [(0, 1), (1, 2), (0, keep)]:
        if first + last <= keep:
            run_select(scores.cuda(), lens, page, keep, first, last)


def test_selection_of_unordered_values(gpu):
    say("select_pages non-finite scores")
    inf, nan = float("inf"), float("nan")
    row = [nan, -inf, 0.0, -0.0, inf, 1e-45, -1e-45, 3e38, -3e38, nan, inf, 0.0, -0.0, -inf, 5.0, -5.0]
    scores = torch.tensor([row, [nan] * 16, [-inf] * 16, [inf] * 16, [-0.0, 0.0] * 8], device="cuda")
    for keep in range(1, 17):
        run_select(scores, [16 * 16] * 5, 16, keep, 0, 1)
        if keep >= 3:
            run_select(scores, [16 * 16 - 3] * 5, 16, keep, 1, 2)


def test_selected_decode_is_attention_over_the_chosen_pages(gpu):
    for layer in ("h16", "h128", "f32"):
        say(f"sparse decode {layer}")
        c = Cache(layer, [1000, 0, 130, 64, 333, 17], 16)
        c.check_means()
        q = c.L.query(6)
        scores = c.scores(q)
        keep = 9
        sel, n = torch.empty(6, keep, dtype=I32, device="cuda"), torch.empty(6, dtype=I32, device="cuda")
        B.select_pages(c.L.dims, scores, c.seq_lens, c.table, c.width, sel, n, keep_first=1, keep_last=2)
        out = torch.empty(6, c.L.h, c.L.dv, dtype=c.L.dtype, device="cuda")
        ws = B.alloc_workspace(B.decode_workspace_size(c.L.dims, 6, keep))
        B.decode(c.L.dims, q, c.L.cache, c.L.ids, c.L.gate, c.L.w_uk, c.L.w_uv, n, sel, keep, ws, out)
        torch.cuda.synchronize()
        cols, tokens = S.select(scores.cpu().numpy(), c.lens, 16, keep, 1, 2)
        t = c.table.cpu().numpy()
        ref = c.L.attend(q, lambda b: c.L.rows(t[b, cols[b]], tokens[b]))
        assert_close(c.L.f64(out), ref, c.L.storage, f"sparse decode {layer}")


def test_captured_step_replays_with_other_lengths(gpu):
    say("page scores and selection captured")
    c = Cache("h16", [600, 300, 0, 64], 16)
    c.check_means()
    q, keep = c.L.query(4), 6
    out = torch.empty(4, c.width, device="cuda")
    sel, n = torch.empty(4, keep, dtype=I32, device="cuda"), torch.empty(4, dtype=I32, device="cuda")
    ws = B.alloc_workspace(B.page_scores_workspace_size(c.L.dims, 4))
    first = c.seq_lens.clone()
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        B.page_scores(c.L.dims, q, c.L.w_uk, c.means, c.seq_lens, c.table, c.width, ws, out)
        B.select_pages(c.L.dims, out, c.seq_lens, c.table, c.width, sel, n)
        B.page_means(c.L.dims, c.L.cache, c.L.ids, c.L.gate, first, c.seq_lens, c.table, c.width, c.means)
    for lens in ([600, 300, 0, 64], [17, 299, 0, 1], [590, 1, 0, 33]):
        c.lens = lens
        c.seq_lens.copy_(cuda_ints(lens))
        first.copy_((c.seq_lens - 20).clamp(min=0))
        eager = c.scores(q)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        cols, tokens = S.select(out.cpu().numpy(), lens, 16, keep, 0, 1)
        assert n.tolist() == tokens
        for b, cs in enumerate(cols):
            assert sel[b, : len(cs)].tolist() == c.table[b].cpu()[cs].tolist()
