"""Operators of a paged EG-MLA server around the decode: what a step does besides attending to every cached token.

A case is a dict of plain values.  Its "kind" names what one pass runs:

  pages   the page table, slots and positions of a step from the request lengths (page_plan), and, where some
          requests have ended, the return of their pages before it (page_release)
  qk      RMSNorm of queries (per head) and keys and the position rotation of both, the key rows written to the
          cache, in one pass (qk_norm_rope)
  shared  decode of a batch whose sequences share a long prefix, the prefix computed once for all (decode_shared)
  scores  the scores of every cached page for each query from the pages' means (page_scores), then the means of the
          pages that the step's tokens changed (page_means)
  select  the pages each query attends to, chosen by score (select_pages), and the decode over them

and, but for "pages", "layer" one of LAYERS (the layers of cases.py).  Sequence lengths are spread evenly over
[min_len, max_len] and handed to the sequences in a random order, so that a case's work does not depend on the seed.

`own` false: elementary torch operations in 32 bits, rounded once at the end.  `own` true: the library's calls.
"""
import math

import numpy as np
import torch

own = False

# heads, head dim (queries and values), latent, RoPE, vocabulary, storage
LAYERS = {
    "tiny": dict(h=4, dh=32, dc=32, dr=0, vocab=1000, dtype="fp32"),
    "f32": dict(h=8, dh=64, dc=128, dr=32, vocab=5000, dtype="fp32"),
    "kv64": dict(h=12, dh=64, dc=64, dr=64, vocab=50304, dtype="bf16"),
    "h16": dict(h=16, dh=128, dc=128, dr=64, vocab=50304, dtype="bf16"),
    "mla320": dict(h=16, dh=128, dc=320, dr=64, vocab=50304, dtype="bf16"),
    "h128": dict(h=128, dh=128, dc=512, dr=64, vocab=129280, dtype="bf16"),
}


def listed():
    return [
        # a decode step of a small batch: one new token for each of 32 sequences, latency only
        dict(name="pages_step_b32", kind="pages", batch=32, page=64, min_len=100, max_len=4000, min_new=1, max_new=1,
             ended=0, short=False),
        # a step of a loaded server: every eighth request has ended and a new prompt takes its place, chunks of
        # prompts for the others
        dict(name="pages_prompt_b256", kind="pages", batch=256, page=64, min_len=0, max_len=3000, min_new=1,
             max_new=401, ended=8, short=False),
        # queries and keys of a decode step, views of one fused projection's rows
        dict(name="qk_step_b8", kind="qk", layer="h16", n=8, q_norm=True, fused=True),
        # those of a prompt of the 128-head layer
        dict(name="qk_prompt_h128", kind="qk", layer="h128", n=4096, q_norm=True, fused=False),
        # the smallest shared decode: a small fp32 layer, a short system prompt
        dict(name="shared_tiny_b4", kind="shared", layer="tiny", batch=4, prefix=128, min_len=1, max_len=100, page=16),
        # the ordinary batch, a long system prompt and short answers
        dict(name="shared_h16_b32", kind="shared", layer="h16", batch=32, prefix=8192, min_len=16, max_len=1000, page=64),
        # many samples of one long document
        dict(name="shared_h16_b256", kind="shared", layer="h16", batch=256, prefix=16384, min_len=1, max_len=512, page=64),
        # the 128-head layer
        dict(name="shared_h128_b64", kind="shared", layer="h128", batch=64, prefix=8000, min_len=50, max_len=1500, page=64),
        # page scores of a decode step, long contexts of mixed length
        dict(name="scores_h16_b32", kind="scores", layer="h16", batch=32, min_len=2000, max_len=32768, new=1, page=64),
        # the same of the 128-head layer, very long contexts, a chunk of new tokens
        dict(name="scores_h128_b8", kind="scores", layer="h128", batch=8, min_len=16384, max_len=65536, new=100, page=64),
        # few sequences of very long context, 4096 tokens kept of up to 65536
        dict(name="select_h16_b8", kind="select", layer="h16", batch=8, min_len=9000, max_len=65536, keep=64, page=64),
        # the 128-head layer, 2048 tokens kept
        dict(name="select_h128_b16", kind="select", layer="h128", batch=16, min_len=1000, max_len=32768, keep=32, page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pages", "qk", "shared", "shared", "scores", "select"])
    page = rng.choice([16, 24, 64, 64, 128])
    if kind == "pages":
        b = _log(rng, 1, 1000)
        lo = rng.choice([0, 1, 17])
        top_new = min(_log(rng, 1, 4000), max(1, 100000 // b))
        return dict(kind=kind, batch=b, page=page, min_len=lo, max_len=lo + _log(rng, 1, max(2, 400000 // b)),
                    min_new=rng.choice([0, 1, top_new]), max_new=top_new, ended=rng.choice([0, 0, 3, 8]),
                    short=rng.random() < 0.3)
    if kind == "qk":
        layer = rng.choice(["tiny", "f32", "kv64", "h16", "mla320", "h128"])
        return dict(kind=kind, layer=layer, n=_log(rng, 1, 4096 if layer == "h128" else 16384),
                    q_norm=rng.random() < 0.5, fused=rng.random() < 0.5)
    if kind == "shared":
        layer = rng.choice(["f32", "kv64", "h16", "h16", "mla320", "h128", "h128"])
        b = _log(rng, 1, {"f32": 32, "kv64": 64, "h16": 256, "mla320": 128, "h128": 64}[layer])
        top = {"f32": 40000, "kv64": 100000, "h16": 4 << 20, "mla320": 1 << 20, "h128": 500000}[layer]
        prefix = min(_log(rng, 1, 32768), top // b)
        hi = _log(rng, 1, min(4000, max(2, 100000 // b)))
        return dict(kind=kind, layer=layer, batch=b, prefix=prefix, min_len=rng.choice([0, 1, hi]), max_len=hi, page=page)
    layer = rng.choice(["f32", "kv64", "h16", "h16", "mla320", "h128"])
    b = _log(rng, 1, 32)
    hi = _log(rng, 100, min(131072, (800000 if layer != "h128" else 300000) // b))
    if kind == "scores":
        return dict(kind=kind, layer=layer, batch=b, min_len=rng.choice([1, hi // 2, hi]), max_len=hi,
                    new=rng.choice([1, 1, rng.randint(2, 300)]), page=page)
    return dict(kind=kind, layer=layer, batch=b, min_len=rng.choice([1, hi // 2, hi]), max_len=hi,
                keep=max(3, min(_log(rng, 3, 300), 8192 // page)), page=page)


def _spread(n, lo, hi):
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


class _Draw:
    """Seeded values on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, shape, dtype, std=1.0, mean=0.0):
        x = torch.randn(shape, generator=self.g, device="cuda")
        if std != 1.0 or mean != 0.0:
            x.mul_(std).add_(mean)
        return x.to(dtype)

    def ints(self, hi, n):
        return torch.randint(0, hi, (n,), generator=self.g, device="cuda", dtype=torch.int32)

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device="cuda").to(torch.int32)

    def spread(self, n, lo, hi):
        return torch.tensor(_spread(n, lo, hi), dtype=torch.int32, device="cuda")[self.perm(n).long()].contiguous()


def _pages_of(lens, page):
    return (lens + (page - 1)) // page


def _table(r, lens, width, page, spare=0):
    """A random page table of `width` columns over ceil(len / page) pages a sequence, -1 behind them; the pages left."""
    per = _pages_of(lens, page)
    n = int(per.sum())
    order = r.perm(n + spare)
    table = torch.full((lens.numel(), width), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(width, device="cuda")[None, :] < per[:, None]] = order[:n]
    return table, order[n:].contiguous()


def _prepare_pages(case, r, s):
    b, page = case["batch"], case["page"]
    cached, new = r.spread(b, case["min_len"], case["max_len"]), r.spread(b, case["min_new"], case["max_new"])
    s["max_tokens"] = sum(_spread(b, case["min_new"], case["max_new"])) + 5
    width = -(-(case["max_len"] + case["max_new"]) // page)
    ended = torch.zeros(b, dtype=torch.int32, device="cuda")
    if case["ended"]:
        ended[:: case["ended"]] = 1
    # free pages: as many as the new tokens can need, or too few of them, and room for all that may come back
    need = sum(-(-x // page) + 1 for x in _spread(b, case["min_new"], case["max_new"]))
    spare = need // 3 if case["short"] else need
    s["table"], free = _table(r, cached, width, page, spare)
    s["free_count"] = torch.tensor([spare], dtype=torch.int32, device="cuda")
    back = torch.full((int(_pages_of(cached, page).sum()) + 1,), -1, dtype=torch.int32, device="cuda")
    s["free"] = torch.cat([free, back])
    s["cached"], s["new"], s["ended"] = cached, new, ended
    s["base"] = torch.full((b,), 77, dtype=torch.int32, device="cuda")  # behind a shared prefix
    i32 = dict(dtype=torch.int32, device="cuda")
    for name, n in (("kept", b), ("lens", b), ("cu", b + 1), ("positions", s["max_tokens"]), ("slots", s["max_tokens"]),
                    ("count_mid", 1), ("count_out", 1)):
        s[name] = torch.zeros(n, **i32)
    return s


def _prepare_qk(case, r, s):
    L, dt, n = s["L"], s["dt"], case["n"]
    h, dq, row = L["h"], L["dh"] + L["dr"], L["dc"] + L["dr"]
    if case["fused"]:
        x = r.normal((n, h * dq + row), dt)
        s["q"], s["kv"] = x[:, : h * dq], x[:, h * dq:]
    else:
        s["q"], s["kv"] = r.normal((n, h * dq), dt), r.normal((n, row), dt)
    s["q_w"] = r.normal((dq,), dt, 0.1, 1.0) if case["q_norm"] else None
    s["k_w"] = r.normal((L["dr"],), dt, 0.1, 1.0) if case["q_norm"] and L["dr"] else None
    s["kv_w"] = r.normal((L["dc"],), dt, 0.1, 1.0)
    s["positions"], s["new_ids"], s["slots"] = r.ints(131072, n), r.ints(L["vocab"], n), r.perm(n + 7)[:n].contiguous()
    s["cache"] = torch.zeros((n + 7, row), dtype=dt, device="cuda")
    s["ids"] = torch.zeros(n + 7, dtype=torch.int32, device="cuda")
    s["q_out"] = torch.empty((n, h, dq), dtype=dt, device="cuda")
    return s


def prepare(case, seed):
    r = _Draw(seed)
    s = dict(kind=case["kind"], case=case)
    if case["kind"] == "pages":
        return _prepare_pages(case, r, s)
    L = LAYERS[case["layer"]]
    dt = torch.bfloat16 if L["dtype"] == "bf16" else torch.float32
    s["L"], s["dt"] = L, dt
    if case["kind"] == "qk":
        return _prepare_qk(case, r, s)
    b, page, h, dh, dc, dr = case["batch"], case["page"], L["h"], L["dh"], L["dc"], L["dr"]
    lens = r.spread(b, case["min_len"], case["max_len"])
    s["lens"], s["max_pages"] = lens, max(1, -(-case["max_len"] // page))
    prefix_pages = -(-case.get("prefix", 0) // page)
    s["table"], s["prefix_table"] = _table(r, lens, s["max_pages"], page, prefix_pages)
    n_pages = int(_pages_of(lens, page).sum()) + prefix_pages
    rows = n_pages * page
    unit = L["dtype"] == "fp32"  # the fp32 layers' values are scaled by their width
    std = 1 / math.sqrt(dc)
    s["w_uk"], s["w_uv"] = r.normal((h, dh, dc), dt, std), r.normal((h, dh, dc), dt, std)
    s["q"] = r.normal((b, h, dh + dr), dt, 1 / math.sqrt(dh) if unit else 1.0)
    s["gate"] = r.normal((L["vocab"], dc), dt, 0.1, 1.0)
    s["cache"] = r.normal((rows, dc + dr), dt, std if unit else 1.0)
    s["ids"] = r.ints(L["vocab"], rows)
    s["out"] = torch.empty((b, h, dh), dtype=dt, device="cuda")
    if case["kind"] == "shared":
        s["prefix_len"] = torch.tensor([case["prefix"]], dtype=torch.int32, device="cuda")
    if case["kind"] == "scores":
        # means as the step before left them: every page's mean over its rows
        s["means"] = _gated(s, torch.arange(rows, device="cuda")).reshape(n_pages, page, dc + dr).mean(1).to(dt)
        s["first"] = (lens - case["new"]).clamp_(min=0)
        s["scores"] = torch.empty((b, s["max_pages"]), dtype=torch.float32, device="cuda")
    if case["kind"] == "select":
        # scores as page_scores gives them: a query's best head over a page's mean key
        s["scores"] = r.normal((b, s["max_pages"]), torch.float32, 0.3, 0.5)
        s["scores"].masked_fill_(torch.arange(s["max_pages"], device="cuda")[None, :] >= _pages_of(lens, page)[:, None],
                                 -math.inf)
        s["sel"] = torch.empty((b, case["keep"]), dtype=torch.int32, device="cuda")
        s["sel_lens"] = torch.empty(b, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _plain_pages(s):
    case, page = s["case"], s["case"]["page"]
    b, width = s["table"].shape
    cached, count, free = s["cached"].long(), s["free_count"].long(), s["free"]
    dev = cached.device
    if case["ended"]:
        gone = s["ended"] != 0
        per = torch.where(gone, _pages_of(cached, page), 0)
        back = torch.arange(width, device=dev)[None, :] < per[:, None]
        at = count + torch.cumsum(back.reshape(-1), 0) - 1
        free = torch.cat([free, free[:1]])  # a place for what is not kept
        free[torch.where(back.reshape(-1), at, free.numel() - 1)] = s["table"].reshape(-1)
        free = free[:-1]
        s["free"].copy_(free)
        count = count + per.sum()
        cached = torch.where(gone, 0, cached)
    new = s["new"].long()
    have, total = _pages_of(cached, page), cached + new
    fits = total <= width * page
    need = torch.where(fits, _pages_of(total, page) - have, 0)
    cu, cn = torch.cumsum(new, 0), torch.cumsum(need, 0)
    served = fits & (cu <= s["max_tokens"]) & ((need == 0) | (cn <= count))
    taken = torch.where(served, need, 0)
    # new entries of the table: the k-th page of a sequence's new ones from the top of the stack
    col = torch.arange(width, device=dev)[None, :]
    fresh = (col >= have[:, None]) & (col < (have + taken)[:, None])
    place = (count - 1 - (cn - need)[:, None] - (col - have[:, None])).clamp(0, free.numel() - 1)
    table = torch.where(fresh, free[place], s["table"])
    cu = torch.cat([cu.new_zeros(1), cu]).clamp(max=s["max_tokens"])
    i = torch.arange(s["max_tokens"], device=dev)
    of = torch.searchsorted(cu[1:], i, right=True)
    inside = of < b
    of = of.clamp(max=b - 1)
    at = cached[of] + i - cu[of]
    positions = torch.where(inside, s["base"][of] + at, 0)
    row = table[of, (at // page).clamp(0, width - 1)].long()
    slots = torch.where(inside & served[of], row * page + at % page, -1)
    lens = torch.where(served, total, cached)
    s["table"].copy_(table)
    return [x.to(torch.int32) for x in (s["table"], s["free"], lens, cu, positions, slots, count - taken.sum())]


def _norm(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()


def _turn(x, positions):
    """Rotation of the adjacent pairs of the last dim; x [n, ..., d_r], the angles in 64 bits."""
    d = x.shape[-1]
    freq = 10000.0 ** (-2.0 * torch.arange(d // 2, device=x.device, dtype=torch.float64) / d)
    angle = (positions.double()[:, None] * freq).reshape([x.shape[0]] + [1] * (x.dim() - 2) + [d // 2])
    cs, sn = torch.cos(angle).float(), torch.sin(angle).float()
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * cs - b * sn, a * sn + b * cs], -1).reshape(x.shape)


def _plain_qk(s):
    L = s["L"]
    dh, dc, n = L["dh"], L["dc"], s["case"]["n"]
    q = _norm(s["q"].reshape(n, L["h"], -1).float(), s["q_w"])
    q = torch.cat([q[..., :dh], _turn(q[..., dh:], s["positions"])], -1)
    kv = s["kv"].float()
    k = _norm(kv[:, dc:], s["k_w"])
    s["cache"][s["slots"].long()] = torch.cat([_norm(kv[:, :dc], s["kv_w"]), _turn(k, s["positions"])], 1).to(s["dt"])
    s["ids"][s["slots"].long()] = s["new_ids"]
    return [q.to(s["dt"]), s["cache"], s["ids"]]


def _gated(s, rows, t=torch.float32):
    """[gated latent | RoPE key] of cache rows, in 32 bits unless asked for more."""
    dc = s["L"]["dc"]
    x = s["cache"][rows].to(t)
    return torch.cat([x[..., :dc] * s["gate"][s["ids"][rows].long()].to(t), x[..., dc:]], -1)


def _absorbed(s):
    """[W_UK^T q^C | q^R] [batch, heads, d_c + d_r], in 32 bits."""
    dh = s["L"]["dh"]
    q = s["q"].float()
    return torch.cat([torch.matmul(q[:, :, :dh].transpose(0, 1), s["w_uk"].float()).transpose(0, 1), q[:, :, dh:]], 2)


def _rows(table, page, n):
    """Cache rows [batch, n] of the first n tokens' places of a page table [batch, pages] (clamped where it ends)."""
    j = torch.arange(n, device=table.device)
    return table.long().clamp(min=0)[:, (j // page).clamp(max=table.shape[1] - 1)] * page + j % page


def _plain_attend(s, lens, table, width, prefix=None):
    """Softmax attention of a batch over its own rows and, in front of them, the shared rows."""
    L, page = s["L"], s["case"]["page"]
    b, h, dc = s["q"].shape[0], L["h"], L["dc"]
    tau = 1 / math.sqrt(L["dh"] + L["dr"])
    qf = _absorbed(s)
    own_key = _gated(s, _rows(table, page, width))
    sc = tau * torch.matmul(qf, own_key.transpose(1, 2))
    sc.masked_fill_(torch.arange(width, device=sc.device)[None, None, :] >= lens[:, None, None], -math.inf)
    top = sc.amax(2, keepdim=True)
    if prefix is not None:
        at, count = prefix
        key = _gated(s, at)
        shared = tau * torch.matmul(qf.reshape(b * h, -1), key.t()).reshape(b, h, -1)
        shared.masked_fill_(torch.arange(key.shape[0], device=sc.device) >= count, -math.inf)
        top = torch.maximum(top, shared.amax(2, keepdim=True))
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(sc - top)
    total, o = p.sum(2, keepdim=True), torch.matmul(p, own_key[..., :dc])
    if prefix is not None:
        p = torch.exp(shared - top)
        total = total + p.sum(2, keepdim=True)
        o = o + torch.matmul(p.reshape(b * h, -1), key[:, :dc]).reshape(b, h, dc)
    o = torch.where(total > 0, o / total, 0.0)
    out = torch.matmul(o.transpose(0, 1), s["w_uv"].float().transpose(1, 2)).transpose(0, 1)
    return out.to(s["dt"])


def _plain_shared(s):
    page = s["case"]["page"]
    at = _rows(s["prefix_table"][None, :], page, s["prefix_table"].numel() * page)[0]
    return _plain_attend(s, s["lens"], s["table"], s["max_pages"] * page, (at, s["prefix_len"]))


def _plain_scores(s):
    L, case, page = s["L"], s["case"], s["case"]["page"]
    tau = 1 / math.sqrt(L["dh"] + L["dr"])
    n = _pages_of(s["lens"], page)
    means = s["means"][s["table"].long().clamp(min=0)].float()
    scores = (tau * torch.matmul(_absorbed(s), means.transpose(1, 2))).amax(1)
    scores.masked_fill_(torch.arange(s["max_pages"], device=n.device)[None, :] >= n[:, None], -math.inf)
    # the pages that the step's tokens changed: at most (new - 1) / page + 2 a sequence
    first = s["first"] // page
    most = (case["new"] - 1) // page + 2
    pg = first[:, None] + torch.arange(most, device=n.device)[None, :]
    change = (pg < n[:, None]) & (s["first"] < s["lens"])[:, None]
    phys = torch.gather(s["table"].long().clamp(min=0), 1, pg.clamp(max=s["max_pages"] - 1).long())
    j = torch.arange(page, device=n.device)
    there = pg[..., None] * page + j < s["lens"][:, None, None]
    # (in 64 bits: a mean is rounded once, to the value that its exact one is nearest to)
    x = _gated(s, phys[..., None] * page + j, torch.float64) * there[..., None]
    mean = (x.sum(2) / there.sum(2).clamp(min=1)[..., None]).to(s["dt"])
    s["means"][phys[change]] = mean[change]
    return [scores, s["means"]]


def _chosen(s):
    """Pages kept, in the order of the sequence: the first one, the last two and the best of the others, ties to the first."""
    keep, page = s["case"]["keep"], s["case"]["page"]
    n = _pages_of(s["lens"], page)[:, None].long()
    j = torch.arange(s["max_pages"], device=n.device)[None, :]
    score = torch.where(torch.isnan(s["scores"]), -math.inf, s["scores"])
    order = torch.sort(score, dim=1, descending=True, stable=True).indices
    always = (j < 1) | (j >= n - 2)
    rank = torch.where(j >= n, 2, torch.where(always, 0, 1))
    order = torch.gather(order, 1, torch.sort(torch.gather(rank, 1, order), dim=1, stable=True).indices)[:, :keep]
    order = torch.sort(torch.where(order < n, order, s["max_pages"]), 1).values
    return torch.nn.functional.pad(order, (0, keep - order.shape[1]), value=s["max_pages"]), n


def _plain_select(s):
    keep, page = s["case"]["keep"], s["case"]["page"]
    order, n = _chosen(s)
    sel = torch.where(order < s["max_pages"], torch.gather(s["table"], 1, order.clamp(max=s["max_pages"] - 1)), -1)
    lens = s["lens"].long() - (n - n.clamp(max=keep))[:, 0] * page
    return [sel.to(torch.int32), lens.to(torch.int32), _plain_attend(s, lens, sel, keep * page)]


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------
def _library():
    from paper_2509_16686_amd import binding
    return binding


def _dims(s):
    L = s["L"]
    lib = _library()
    return lib.make_dims(num_heads=L["h"], head_dim=L["dh"], v_head_dim=L["dh"], latent_dim=L["dc"], rope_dim=L["dr"],
                         vocab_size=L["vocab"], page_size=s["case"].get("page", 64),
                         dtype=lib.BF16 if L["dtype"] == "bf16" else lib.FP32)


def _own_pages(s):
    lib, case = _library(), s["case"]
    cached, count = s["cached"], s["free_count"]
    if case["ended"]:
        lib.page_release(case["page"], s["cached"], s["ended"], s["table"], s["free"], s["free_count"], s["kept"],
                         s["count_mid"])
        cached, count = s["kept"], s["count_mid"]
    lib.page_plan(case["page"], cached, s["new"], s["table"], s["free"], count, s["lens"], s["cu"], s["positions"],
                  s["slots"], s["count_out"], position_base=s["base"])
    return [s["table"], s["free"], s["lens"], s["cu"], s["positions"], s["slots"], s["count_out"]]


def _own_qk(s):
    lib = _library()
    if "dims" not in s:
        s["dims"] = _dims(s)
    lib.qk_norm_rope(s["dims"], s["q"], s["q_out"], s["kv"], s["cache"], s["ids"], s["new_ids"], s["positions"],
                     s["slots"], q_norm_w=s["q_w"], kv_norm_w=s["kv_w"], k_norm_w=s["k_w"])
    return [s["q_out"], s["cache"], s["ids"]]


def _own_shared(s):
    lib = _library()
    if "dims" not in s:
        s["dims"] = _dims(s)
        s["ws"] = lib.alloc_workspace(lib.decode_shared_workspace_size(s["dims"], s["case"]["batch"], s["max_pages"],
                                                                       s["prefix_table"].numel()))
    lib.decode_shared(s["dims"], s["q"], s["cache"], s["ids"], s["gate"], s["w_uk"], s["w_uv"], s["prefix_len"],
                      s["prefix_table"], s["lens"], s["table"], s["max_pages"], s["ws"], s["out"])
    return s["out"]


def _own_scores(s):
    lib = _library()
    if "dims" not in s:
        s["dims"] = _dims(s)
        s["ws"] = lib.alloc_workspace(lib.page_scores_workspace_size(s["dims"], s["case"]["batch"]))
    lib.page_scores(s["dims"], s["q"], s["w_uk"], s["means"], s["lens"], s["table"], s["max_pages"], s["ws"], s["scores"])
    lib.page_means(s["dims"], s["cache"], s["ids"], s["gate"], s["first"], s["lens"], s["table"], s["max_pages"], s["means"])
    return [s["scores"], s["means"]]


def _own_select(s):
    lib, keep = _library(), s["case"]["keep"]
    if "dims" not in s:
        s["dims"] = _dims(s)
        s["ws"] = lib.alloc_workspace(lib.decode_workspace_size(s["dims"], s["case"]["batch"], keep))
    lib.select_pages(s["dims"], s["scores"], s["lens"], s["table"], s["max_pages"], s["sel"], s["sel_lens"], keep_first=1,
                     keep_last=2)
    lib.decode(s["dims"], s["q"], s["cache"], s["ids"], s["gate"], s["w_uk"], s["w_uv"], s["sel_lens"], s["sel"], keep,
               s["ws"], s["out"])
    return [s["sel"], s["sel_lens"], s["out"]]


PLAIN = dict(pages=_plain_pages, qk=_plain_qk, shared=_plain_shared, scores=_plain_scores, select=_plain_select)
OWN = dict(pages=_own_pages, qk=_own_qk, shared=_own_shared, scores=_own_scores, select=_own_select)


def run(s):
    if own:
        return OWN[s["kind"]](s)
    return PLAIN[s["kind"]](s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "pages":
        b, page = case["batch"], case["page"]
        new, lens = sum(_spread(b, case["min_new"], case["max_new"])), sum(_spread(b, case["min_len"], case["max_len"]))
        back = lens // case["ended"] // page if case["ended"] else 0
        # lengths in and out, offsets, position and slot of each token, the entries of new and returned pages
        return {"bytes": 4 * (6 * b + 2 * new + 2 * (new // page + 1) + 2 * back), "flops": 4 * new}
    L = LAYERS[case["layer"]]
    h, dh, dc, dr, v = L["h"], L["dh"], L["dc"], L["dr"], L["vocab"]
    eb = 2 if L["dtype"] == "bf16" else 4
    if kind == "qk":
        n = case["n"]
        return {"bytes": n * (2 * (h * (dh + dr) + dc + dr) * eb + 16), "flops": n * (4 * (h * (dh + dr) + dc + dr) + 3 * (h + 1) * dr)}
    b, page = case["batch"], case["page"]
    lens = _spread(b, case["min_len"], case["max_len"])
    query = b * h * (dh + dr) * eb
    weight = h * dh * dc * eb
    absorb = 2 * b * h * dh * dc

    def attend(n, pairs):  # n cached tokens, `pairs` (query row, token) pairs
        gates = v * (1 - (1 - 1 / v) ** n) * dc * eb
        return n * ((dc + dr) * eb + 4) + gates + query + 2 * weight + b * h * dh * eb, 2 * absorb + pairs * 2 * (2 * dc + dr)

    if kind == "shared":
        by, fl = attend(sum(lens) + case["prefix"], (sum(lens) + b * case["prefix"]) * h)
    elif kind == "scores":
        pages = sum(-(-x // page) for x in lens)
        change = [(-(-x // page)) - max(0, x - case["new"]) // page for x in lens]
        rows = sum(min(x, c * page) for x, c in zip(lens, change))
        by = query + weight + pages * (dc + dr) * eb + 4 * b * -(-case["max_len"] // page)
        by += rows * ((2 * dc + dr) * eb + 4) + sum(change) * (dc + dr) * eb
        fl = absorb + pages * h * 2 * (dc + dr) + rows * (2 * dc + dr)
    else:
        kept = sum(min(x, case["keep"] * page) for x in lens)
        by, fl = attend(kept, kept * h)
        by += 4 * sum(-(-x // page) for x in lens)
    return {"bytes": int(by), "flops": int(fl)}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_pages(s):
    """The serving rules one sequence after the other, on the host."""
    case, page = s["case"], s["case"]["page"]
    table, free = s["table"].cpu().numpy().copy(), s["free"].cpu().numpy().copy()
    cached, new, base = (s[k].cpu().numpy().astype(np.int64) for k in ("cached", "new", "base"))
    ended, count = s["ended"].cpu().numpy(), int(s["free_count"])
    b, width = table.shape
    if case["ended"]:
        for i in np.flatnonzero(ended):
            n = -(-cached[i] // page)
            free[count:count + n] = table[i, :n]
            count, cached[i] = count + n, 0
    lens, cu = cached.copy(), np.zeros(b + 1, dtype=np.int64)
    positions, slots = np.zeros(s["max_tokens"], dtype=np.int64), np.full(s["max_tokens"], -1, dtype=np.int64)
    closed = False  # a sequence that finds too few pages ends the giving of pages
    for i in range(b):
        cu[i + 1] = min(cu[i] + new[i], s["max_tokens"])
        have, want = -(-cached[i] // page), -(-(cached[i] + new[i]) // page)
        t = cached[i] + np.arange(cu[i + 1] - cu[i])
        positions[cu[i]:cu[i + 1]] = base[i] + t
        if want > width or cu[i] + new[i] > s["max_tokens"]:
            continue
        closed = closed or want - have > count
        if closed and want > have:
            continue
        for p in range(have, want):
            count -= 1
            table[i, p] = free[count]
        lens[i] += new[i]
        slots[cu[i]:cu[i + 1]] = table[i, t // page].astype(np.int64) * page + t % page
    return [torch.from_numpy(np.asarray(x, dtype=np.int32)) for x in (table, free, lens, cu, positions, slots, [count])]


def _exact_norm(x, w):
    return x if w is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.double()


def _exact_qk(s):
    L = s["L"]
    dh, dc, dr, n = L["dh"], L["dc"], L["dr"], s["case"]["n"]
    angle = s["positions"].double()[:, None] * torch.exp(-torch.arange(0, dr, 2, device="cuda").double() / max(dr, 1) * math.log(10000.0))
    turn = torch.polar(torch.ones_like(angle), angle)

    def rotated(x):  # pairs as complex numbers
        z = torch.view_as_complex(x.reshape(n, -1, dr // 2, 2).contiguous()) * turn[:, None, :]
        return torch.view_as_real(z).reshape(x.shape)

    q = _exact_norm(s["q"].double().reshape(n, L["h"], dh + dr), s["q_w"])
    kv = s["kv"].double()
    k = _exact_norm(kv[:, dc:], s["k_w"])
    if dr:
        q, k = torch.cat([q[..., :dh], rotated(q[..., dh:])], -1), rotated(k)
    cache, ids = s["cache"].double(), s["ids"].clone()
    cache[s["slots"].long()] = torch.cat([_exact_norm(kv[:, :dc], s["kv_w"]), k], 1)
    ids[s["slots"].long()] = s["new_ids"]
    return [q, cache, ids]


def _exact_rows(s, pages, n):
    at = (pages.long()[:, None] * s["case"]["page"] + torch.arange(s["case"]["page"], device="cuda")).reshape(-1)[:n]
    x, dc = s["cache"][at].double(), s["L"]["dc"]
    return torch.cat([x[:, :dc] * s["gate"][s["ids"][at].long()].double(), x[:, dc:]], 1)


def _exact_query(s, b):
    dh = s["L"]["dh"]
    q = s["q"][b].double()
    return torch.cat([(q[:, None, :dh] @ s["w_uk"].double())[:, 0], q[:, dh:]], 1) / math.sqrt(dh + s["L"]["dr"])


def _exact_attend(s, rows_of):
    dc = s["L"]["dc"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b in range(out.shape[0]):
        key = rows_of(b)
        if key.shape[0]:
            o = torch.softmax(_exact_query(s, b) @ key.T, 1) @ key[:, :dc]
            out[b] = (s["w_uv"].double() @ o[:, :, None])[:, :, 0]
    return out


def _exact_shared(s):
    shared, lens = _exact_rows(s, s["prefix_table"], s["case"]["prefix"]), s["lens"].tolist()
    return _exact_attend(s, lambda b: torch.cat([shared, _exact_rows(s, s["table"][b].clamp(min=0), lens[b])]))


def _exact_scores(s):
    page, lens, first = s["case"]["page"], s["lens"].tolist(), s["first"].tolist()
    scores = torch.full(s["scores"].shape, -math.inf, dtype=torch.float64, device="cuda")
    means = s["means"].double()
    for b, n in enumerate(lens):
        pages = s["table"][b, : -(-n // page)].long()
        scores[b, : pages.numel()] = (_exact_query(s, b) @ s["means"][pages].double().T).amax(0)
        if first[b] < n:
            for p in range(first[b] // page, -(-n // page)):
                means[pages[p]] = _exact_rows(s, pages[p:p + 1], min(page, n - p * page)).mean(0)
    return [scores, means]


def _exact_select(s):
    keep, page, lens = s["case"]["keep"], s["case"]["page"], s["lens"].tolist()
    scores, table = s["scores"].cpu().numpy(), s["table"].cpu().numpy()
    sel, sel_lens = np.full((len(lens), keep), -1, dtype=np.int32), np.zeros(len(lens), dtype=np.int32)
    for b, n in enumerate(lens):
        have = -(-n // page)
        others = [p for p in range(1, have - 2)]
        always = [p for p in range(have) if p not in range(1, have - 2)]
        others.sort(key=lambda p: (-scores[b, p], p))
        pages = sorted(always + others[: keep - len(always)])
        sel[b, : len(pages)] = table[b, pages]
        sel_lens[b] = n - (have - len(pages)) * page
    out = _exact_attend(s, lambda b: _exact_rows(s, torch.from_numpy(sel[b]).cuda().clamp(min=0), int(sel_lens[b])))
    return [torch.from_numpy(sel), torch.from_numpy(sel_lens), out]


EXACT = dict(pages=_exact_pages, qk=_exact_qk, shared=_exact_shared, scores=_exact_scores, select=_exact_select)


def exact(case, seed):
    return EXACT[case["kind"]](prepare(case, seed))
