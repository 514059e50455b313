"""Operators of a quantised latent cache: rotation of query rows, key rows written in 8 bits, read back, and attended to.

The cache of these operators holds, for each token, the gated latent c (.) G[id] as e4m3 codes with one power of two for
the row (a byte: 127 plus the exponent) and the RoPE key in bf16 behind the codes.  A case is a dict of plain values; its
"kind" names what one pass runs:

  rope    rotation of the RoPE part of query rows, pairs adjacent or half a part away, with plain frequencies or those of
          a stretched context; forward, or the gradient's way back (rope_rows)
  write   norm, gate and rotation of the key rows of a step's tokens, written to their slots in 8 bits (quant_write), and the
          same tokens read back, packed by sequence (quant_read)
  read    cached sequences read back (quant_read)
  attend  attention of the new tokens of each sequence, causal among themselves, over the cache: one new token a
          sequence (decode), or several (a chunk of a prompt, drafted tokens to verify) (quant_attend)

and "layer" one of LAYERS.  Lengths are spread evenly over [min_len, max_len] and handed out in a random order; "min_new"
and "max_new" are the new tokens of a sequence, among its length.

`own` false: elementary torch operations in 32 bits, rounded once at the end.  `own` true: the library's calls.
"""
import math

import torch

own = False

# heads, head dim (queries and values), latent, RoPE, vocabulary
LAYERS = {
    "odd": dict(h=5, dh=40, dc=48, dr=24, vocab=1000),
    "kv64": dict(h=12, dh=64, dc=64, dr=64, vocab=50304),
    "h16": dict(h=16, dh=128, dc=128, dr=64, vocab=50304),
    "mla320": dict(h=16, dh=128, dc=320, dr=64, vocab=50304),
    "h128": dict(h=128, dh=128, dc=512, dr=64, vocab=129280),
}
THETA, TRAINED = 10000.0, 4096  # base of the frequencies; positions that a stretched layer was trained on
TOP = 448.0                     # largest e4m3 value


def listed():
    return [
        # query rows of a decode step, views of a fused projection's rows: latency only
        dict(name="rope_step_b8", kind="rope", layer="h16", n=8, dtype="bf16", half=True, factor=1.0, back=False, fused=True),
        # gradient of the query rows of a long training sequence of the 128-head layer, its context stretched
        dict(name="rope_back_h128", kind="rope", layer="h128", n=8192, dtype="bf16", half=False, factor=8.0, back=True,
             fused=False),
        # one new token for each of 32 sequences
        dict(name="write_step_b32", kind="write", layer="h16", batch=32, min_len=100, max_len=4000, min_new=1, max_new=1,
             page=64, norm=True, half=False, factor=1.0),
        # prompts of the 128-head layer, of different lengths
        dict(name="write_prompt_h128", kind="write", layer="h128", batch=8, min_len=3000, max_len=5000, min_new=100,
             max_new=3000, page=64, norm=True, half=True, factor=8.0),
        # a few short requests taken up again
        dict(name="read_h16_b4", kind="read", layer="h16", batch=4, min_len=100, max_len=2000, page=64),
        # long documents of the 128-head layer
        dict(name="read_h128_b16", kind="read", layer="h128", batch=16, min_len=1000, max_len=32768, page=64),
        # the smallest decode: a small layer of odd sizes, contexts of 1 to 70 tokens, small pages
        dict(name="decode_odd_b3", kind="attend", layer="odd", batch=3, min_len=1, max_len=70, min_new=1, max_new=1, page=16),
        # the ordinary decode batch, equal contexts
        dict(name="decode_h16_b32", kind="attend", layer="h16", batch=32, min_len=4096, max_len=4096, min_new=1, max_new=1,
             page=64),
        # a loaded server, mixed contexts
        dict(name="decode_h16_b256", kind="attend", layer="h16", batch=256, min_len=250, max_len=8192, min_new=1, max_new=1,
             page=64),
        # the 128-head layer, mixed contexts
        dict(name="decode_h128_b64", kind="attend", layer="h128", batch=64, min_len=512, max_len=16384, min_new=1, max_new=1,
             page=64),
        # chunks of prompts over what is cached of them
        dict(name="chunk_h16_b8", kind="attend", layer="h16", batch=8, min_len=600, max_len=8192, min_new=200, max_new=600,
             page=64),
        # drafted tokens of the 128-head layer to verify
        dict(name="verify_h128_b16", kind="attend", layer="h128", batch=16, min_len=2000, max_len=16000, min_new=4, max_new=4,
             page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["rope", "write", "read", "attend", "attend", "attend"])
    layer = rng.choice(["odd", "kv64", "h16", "h16", "mla320", "h128"])
    L = LAYERS[layer]
    page, half, factor = rng.choice([16, 24, 64, 64, 128]), rng.random() < 0.5, rng.choice([1.0, 4.0, 40.0])
    if kind == "rope":
        return dict(kind=kind, layer=layer, n=_log(rng, 1, 8192 if layer == "h128" else 16384),
                    dtype=rng.choice(["bf16", "bf16", "fp32"]), half=half, factor=factor, back=rng.random() < 0.4,
                    fused=rng.random() < 0.5)
    if kind == "write":
        batch, top = _log(rng, 1, 64), rng.choice([1, _log(rng, 1, 3000)])
        top = min(top, 12000 // batch)
        return dict(kind=kind, layer=layer, batch=batch, min_len=top, max_len=top + _log(rng, 1, 4000),
                    min_new=rng.choice([1, top]), max_new=top, page=page, norm=rng.random() < 0.6, half=half, factor=factor)
    if kind == "read":
        batch = _log(rng, 1, 64)
        hi = _log(rng, 1, 250000 // batch)
        return dict(kind=kind, layer=layer, batch=batch, min_len=rng.choice([0, 1, hi]), max_len=hi, page=page)
    new = rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 600)])
    batch = _log(rng, 1, 256 if new == 1 else 32)
    # (query row, token) pairs and cached tokens of the largest listed cases
    pairs = int(6e10 / (2 * L["dc"] + L["dr"])) // (new * L["h"])
    hi = _log(rng, new, max(new, min(65536, 1000000 // batch, pairs // batch)))
    return dict(kind=kind, layer=layer, batch=batch, min_len=rng.choice([new, max(new, hi // 8), hi]), max_len=hi,
                min_new=rng.choice([1, new]), max_new=new, page=page)


def _spread(n, lo, hi):
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _lens(case):
    return _spread(case["batch"], case["min_len"], case["max_len"])


def _news(case):
    return _spread(case["batch"], case["min_new"], case["max_new"])


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
        return torch.randperm(n, generator=self.g, device="cuda")


def _pages_of(lens, page):
    return (lens + (page - 1)) // page


def _prepare_rope(case, r, s):
    L, n = s["L"], case["n"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    h, dq = L["h"], L["dh"] + L["dr"]
    x = r.normal((n, h * dq + (L["dc"] + L["dr"] if case["fused"] else 0)), dt)
    s["x"] = x[:, : h * dq].reshape(n, h, dq) if not case["fused"] else x[:, : h * dq].unflatten(1, (h, dq))
    s["positions"] = r.ints(int(TRAINED * case["factor"]), n)
    s["out"] = torch.empty((n, h, dq), dtype=dt, device="cuda")
    return s


def prepare(case, seed):
    r = _Draw(seed)
    L = LAYERS[case["layer"]]
    s = dict(kind=case["kind"], case=case, L=L)
    if case["kind"] == "rope":
        return _prepare_rope(case, r, s)
    b, page, h, dh, dc, dr = case["batch"], case["page"], L["h"], L["dh"], L["dc"], L["dr"]
    bf = torch.bfloat16
    order = r.perm(b)
    lens = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")[order].contiguous()
    s["lens"], s["width"] = lens, max(1, -(-case["max_len"] // page))
    per = _pages_of(lens, page)
    n_pages = sum(-(-x // page) for x in _lens(case)) + 1
    table = torch.full((b, s["width"]), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(s["width"], device="cuda")[None, :] < per[:, None]] = r.perm(n_pages)[1:].to(torch.int32)
    s["table"], rows = table, n_pages * page
    if case["kind"] == "read":
        new = lens
        s["first"] = None
        s["total"] = sum(_lens(case))
    else:
        new = torch.tensor(_news(case), dtype=torch.int32, device="cuda")[r.perm(b)].contiguous().minimum(lens)
        s["first"] = lens - new
        s["total"] = sum(_news(case))  # (min_len >= max_new: none is cut)
    s["new"] = new
    s["cu"] = torch.cat([new.new_zeros(1), torch.cumsum(new, 0).to(torch.int32)])
    s["codes"] = torch.zeros((rows, dc + 2 * dr), dtype=torch.uint8, device="cuda")
    s["scales"] = torch.full((rows,), 127, dtype=torch.uint8, device="cuda")
    if case["kind"] == "write":
        n = s["total"]
        x = r.normal((n, h * (dh + dr) + dc + dr), bf) if n <= 256 else r.normal((n, dc + dr), bf)
        s["kv"] = x[:, -(dc + dr):]  # of a step: a view of the fused projection's rows
        s["kv_w"] = r.normal((dc,), bf, 0.1, 1.0) if case["norm"] else None
        s["k_w"] = r.normal((dr,), bf, 0.1, 1.0) if case["norm"] else None
        s["gate"] = r.normal((L["vocab"], dc), bf, 0.1, 1.0)
        s["ids"] = r.ints(L["vocab"], n)
        of = torch.repeat_interleave(torch.arange(b, device="cuda"), new.long())
        at = torch.arange(n, device="cuda") - s["cu"][of] + s["first"][of]
        s["positions"] = at.to(torch.int32)
        s["slots"] = (table[of, at // page] * page + at % page).to(torch.int32)
    else:
        # what quant_write leaves: gated latents near one, quantised, and RoPE keys
        c = r.normal((rows, dc), torch.float32) * r.normal((rows, 1), torch.float32, 0.3, 1.0)
        codes, s["scales"] = _quantise(c)
        s["codes"][:, :dc] = codes.view(torch.uint8)
        s["codes"][:, dc:] = r.normal((rows, dr), bf).view(torch.uint8)
    if case["kind"] != "attend":
        s["out"] = torch.empty((s["total"], dc + dr), dtype=bf, device="cuda")
        return s
    std = 1 / math.sqrt(dc)
    s["w_uk"], s["w_uv"] = r.normal((h, dh, dc), bf, std), r.normal((h, dh, dc), bf, std)
    s["q"] = r.normal((s["total"], h, dh + dr), bf)
    s["out"] = torch.empty((s["total"], h, dh), dtype=bf, device="cuda")
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------
def _frequencies(dr, factor):
    """Radians a position of each pair; of a context stretched `factor` times: pairs that turn fewer times than once over
    the trained positions are slowed by it, those of 32 turns or more are not, the others in between."""
    f = THETA ** (-2.0 * torch.arange(dr // 2, device="cuda", dtype=torch.float64) / dr)
    if factor == 1.0:
        return f
    keep = ((f * (TRAINED / (2 * math.pi)) - 1.0) / 31.0).clamp(0.0, 1.0)
    return f * (keep + (1.0 - keep) / factor)


def _magnitude(factor):
    return 1.0 if factor == 1.0 else 0.1 * math.log(factor) + 1.0


def _turn(x, positions, half, factor, back=False):
    """Rotation of the last dim of x [n, ..., d_r]; the angles in 64 bits."""
    d = x.shape[-1]
    angle = positions.double()[:, None] * _frequencies(d, factor) * (-1.0 if back else 1.0)
    angle = angle.reshape([x.shape[0]] + [1] * (x.dim() - 2) + [d // 2])
    cs, sn = (torch.cos(angle) * _magnitude(factor)).float(), (torch.sin(angle) * _magnitude(factor)).float()
    a, b = (x[..., : d // 2], x[..., d // 2:]) if half else (x[..., 0::2], x[..., 1::2])
    u, v = a * cs - b * sn, a * sn + b * cs
    return torch.cat([u, v], -1) if half else torch.stack([u, v], -1).reshape(x.shape)


def _plain_rope(s):
    case, dh = s["case"], s["L"]["dh"]
    x = s["x"].float()
    part = _turn(x[..., dh:], s["positions"], case["half"], case["factor"], case["back"])
    return torch.cat([x[..., :dh], part], -1).to(s["x"].dtype)


def _quantise(c):
    """e4m3 codes of rows and their scale bytes: the smallest power of two that brings the row within the codes' range."""
    m, e = torch.frexp(c.abs().amax(1) / TOP)
    e = torch.where(m == 0, 0, e - (m == 0.5).to(e.dtype)).clamp(-126, 120)
    return torch.ldexp(c, -e[:, None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(s, rows):
    """[gated latent | RoPE key] of cache rows in 32 bits."""
    dc = s["L"]["dc"]
    x = s["codes"][rows]
    c = torch.ldexp(x[..., :dc].contiguous().view(torch.float8_e4m3fn).float(), s["scales"][rows][..., None].int() - 127)
    return torch.cat([c, x[..., dc:].contiguous().view(torch.bfloat16).float()], -1)


def _norm(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()


def _packed(s):
    """Cache rows of the tokens that are read, packed by sequence."""
    page = s["case"]["page"]
    i = torch.arange(s["total"], device="cuda")
    of = torch.searchsorted(s["cu"][1:].long(), i, right=True)
    at = i - s["cu"][of] + (0 if s["first"] is None else s["first"][of])
    return s["table"][of, at // page].long() * page + at % page


def _plain_read(s):
    return _values(s, _packed(s)).to(torch.bfloat16)


def _plain_write(s):
    case, dc = s["case"], s["L"]["dc"]
    kv = s["kv"].float()
    c = _norm(kv[:, :dc], s["kv_w"]) * s["gate"][s["ids"].long()].float()
    k = _turn(_norm(kv[:, dc:], s["k_w"]), s["positions"], case["half"], case["factor"])
    codes, scales = _quantise(c)
    at = s["slots"].long()
    s["codes"][at] = torch.cat([codes.view(torch.uint8), k.to(torch.bfloat16).view(torch.uint8)], 1)
    s["scales"][at] = scales
    return _plain_read(s)


def _plain_attend(s):
    L, case, page = s["L"], s["case"], s["case"]["page"]
    b, h, dh, dc, most = case["batch"], L["h"], L["dh"], L["dc"], case["max_new"]
    q = s["q"].float()
    qf = torch.matmul(q[:, :, :dh].transpose(0, 1), s["w_uk"].float()).transpose(0, 1)
    qf = torch.cat([qf, q[:, :, dh:]], 2) / math.sqrt(dh + L["dr"])
    # the new tokens of each sequence side by side
    i = torch.arange(most, device="cuda")
    there = i[None, :] < s["new"][:, None]
    row = torch.where(there, s["cu"][:-1, None] + i, 0).long()
    j = torch.arange(s["width"] * page, device="cuda")
    key = _values(s, s["table"].long().clamp(min=0)[:, j // page] * page + j % page)
    sc = torch.matmul(qf[row].reshape(b, most * h, -1), key.transpose(1, 2)).reshape(b, most, h, -1)
    last = s["first"][:, None] + i  # a new token's own place: the last one it attends to
    sc.masked_fill_(j > last[:, :, None, None], -math.inf)
    p = torch.exp(sc - sc.amax(3, keepdim=True))
    del sc
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p.reshape(b, most * h, -1), key[..., :dc]).reshape(b, most, h, dc) / total
    o = o[there]  # packed again
    return torch.matmul(o.transpose(0, 1), s["w_uv"].float().transpose(1, 2)).transpose(0, 1).to(torch.bfloat16)


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------
def _library():
    from paper_2509_16686_amd import binding
    return binding


def _keep(s):
    """Layer shapes, rotation and workspace, as a program keeps them."""
    if "dims" in s:
        return _library()
    lib, L, case = _library(), s["L"], s["case"]
    s["dims"] = lib.make_dims(num_heads=L["h"], head_dim=L["dh"], v_head_dim=L["dh"], latent_dim=L["dc"], rope_dim=L["dr"],
                              vocab_size=L["vocab"], page_size=case.get("page", 64), dtype=lib.BF16)
    if "half" in case:
        freq = None if case["factor"] == 1.0 else lib.rope_frequencies(L["dr"], case["factor"], TRAINED, theta=THETA)
        s["rope"] = lib.make_rope(layout=lib.ROPE_HALF if case["half"] else lib.ROPE_PAIRS, theta=THETA, frequencies=freq,
                                  magnitude=_magnitude(case["factor"]))
    if case["kind"] == "attend":
        s["ws"] = lib.alloc_workspace(lib.quant_attend_workspace_size(s["dims"], case["batch"], s["total"], s["width"]))
    return lib


def _own_rope(s):
    lib = _keep(s)
    lib.rope_rows(s["rope"], s["x"], s["positions"], s["out"], rope_dim=s["L"]["dr"], inverse=s["case"]["back"])
    return s["out"]


def _own_read(s):
    lib = _keep(s)
    lib.quant_read(s["dims"], s["codes"], s["scales"], s["first"], s["cu"], s["table"], s["out"])
    return s["out"]


def _own_write(s):
    lib = _keep(s)
    lib.quant_write(s["dims"], s["rope"], s["kv"], s["positions"], s["slots"], s["codes"], s["scales"], gate_table=s["gate"],
                 token_ids=s["ids"], kv_norm_w=s["kv_w"], k_norm_w=s["k_w"])
    return _own_read(s)


def _own_attend(s):
    lib = _keep(s)
    lib.quant_attend(s["dims"], s["q"], None if s["case"]["max_new"] == 1 else s["cu"], s["codes"], s["scales"], s["w_uk"],
                  s["w_uv"], s["lens"], s["table"], s["width"], s["ws"], s["out"])
    return s["out"]


PLAIN = dict(rope=_plain_rope, write=_plain_write, read=_plain_read, attend=_plain_attend)
OWN = dict(rope=_own_rope, write=_own_write, read=_own_read, attend=_own_attend)


def run(s):
    return (OWN if own else PLAIN)[s["kind"]](s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    kind, L = case["kind"], LAYERS[case["layer"]]
    h, dh, dc, dr, v = L["h"], L["dh"], L["dc"], L["dr"], L["vocab"]
    row, wide = dc + 2 * dr + 1, 2 * (dc + dr)  # bytes of a cached token, of its values in bf16
    if kind == "rope":
        n = case["n"]
        return {"bytes": n * (2 * h * (dh + dr) * (2 if case["dtype"] == "bf16" else 4) + 4), "flops": n * h * 3 * dr}
    b, lens = case["batch"], sorted(_lens(case))
    if kind == "read":
        n = sum(lens)
        return {"bytes": n * (row + wide) + 4 * (2 * b + sum(-(-x // case["page"]) for x in lens)), "flops": n * dc}
    new = _news(case)
    n = sum(new)
    if kind == "write":
        gates = v * (1 - (1 - 1 / v) ** n) * 2 * dc
        return {"bytes": int(n * (2 * wide + 2 * row + 12) + gates), "flops": n * (8 * dc + 8 * dr)}
    # lengths and new tokens meet in a random order: the pairs as they are on average
    pairs = sum((sum(lens) / b - (x - 1) / 2) * x for x in new) * h
    by = sum(lens) * row + n * h * 2 * (2 * dh + dr) + 4 * h * dh * dc + 4 * sum(-(-x // case["page"]) for x in lens)
    return {"bytes": int(by), "flops": int(4 * n * h * dh * dc + pairs * 2 * (2 * dc + dr))}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_turn(x, positions, case, back=False):
    """Pairs as complex numbers, times e^(i angle) and the magnitude; x [n, heads, d_r]."""
    n, h, d = x.shape
    f = [math.exp(-2.0 * m / d * math.log(THETA)) for m in range(d // 2)]
    if case["factor"] != 1.0:
        for m in range(d // 2):
            turns = TRAINED * f[m] / (2 * math.pi)
            slow = 1.0 if turns <= 1 else 0.0 if turns >= 32 else (32 - turns) / 31
            f[m] = slow * f[m] / case["factor"] + (1 - slow) * f[m]
    angle = positions.double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    size = torch.full_like(angle, 1.0 if case["factor"] == 1.0 else 1.0 + math.log(case["factor"]) / 10)
    turn = torch.polar(size, -angle if back else angle)[:, None, :]
    z = x.reshape(n, h, 2, d // 2).transpose(2, 3) if case["half"] else x.reshape(n, h, d // 2, 2)
    y = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
    return (y.transpose(2, 3) if case["half"] else y).reshape(n, h, d)


def _exact_rope(s):
    dh = s["L"]["dh"]
    x = s["x"].double()
    return torch.cat([x[..., :dh], _exact_turn(x[..., dh:], s["positions"], s["case"], s["case"]["back"])], 2)


def _exact_row(s, at):
    """The values of cache rows, decoded bit by bit: sign, exponent and fraction of a code, the row's power of two."""
    dc = s["L"]["dc"]
    x = s["codes"][at]
    code = x[:, :dc].to(torch.int64)
    exponent, fraction = (code >> 3) & 15, (code & 7).double()
    size = torch.where(exponent == 0, fraction / 8 * 2.0 ** -6, (1 + fraction / 8) * 2.0 ** (exponent - 7).double())
    c = torch.where(code >= 128, -size, size) * 2.0 ** (s["scales"][at].double() - 127)[:, None]
    return torch.cat([c, x[:, dc:].contiguous().view(torch.bfloat16).double()], 1)


def _exact_places(s, b, lo, hi):
    j = torch.arange(lo, hi, device="cuda")
    return s["table"][b].long()[j // s["case"]["page"]] * s["case"]["page"] + j % s["case"]["page"]


def _exact_read(s):
    lens, new = s["lens"].tolist(), s["new"].tolist()
    return torch.cat([_exact_row(s, _exact_places(s, b, n - k, n)) for b, (n, k) in enumerate(zip(lens, new))])


def _exact_write(s):
    dc = s["L"]["dc"]
    c, k = s["kv"].double().split([dc, s["L"]["dr"]], 1)
    if s["kv_w"] is not None:
        c = c / torch.sqrt(c.square().sum(1, keepdim=True) / dc + 1e-6) * s["kv_w"].double()
        k = k / torch.sqrt(k.square().sum(1, keepdim=True) / s["L"]["dr"] + 1e-6) * s["k_w"].double()
    c = c * s["gate"].double()[s["ids"].long()]
    k = _exact_turn(k[:, None, :], s["positions"], s["case"])[:, 0]
    top = c.abs().amax(1, keepdim=True)
    scale = torch.where(top > 0, 2.0 ** torch.ceil(torch.log2(top / TOP)), 1.0)
    x = c / scale
    step = 2.0 ** (torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)  # of the codes around a value
    return torch.cat([torch.round(x / step) * step * scale, k], 1)  # slots go in the order of the tokens


def _exact_attend(s):
    L = s["L"]
    dh, dc = L["dh"], L["dc"]
    lens, cu = s["lens"].tolist(), s["cu"].tolist()
    w_uk, w_uv = s["w_uk"].double(), s["w_uv"].double()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        key = _exact_row(s, _exact_places(s, b, 0, n))
        k = cu[b + 1] - cu[b]
        for i0 in range(0, k, 32):  # some rows at a time
            i1 = min(k, i0 + 32)
            q = s["q"][cu[b] + i0:cu[b] + i1].double()
            q = torch.cat([torch.stack([q[:, h, :dh] @ w_uk[h] for h in range(L["h"])], 1), q[:, :, dh:]], 2)
            sc = (q.reshape(-1, dc + L["dr"]) @ key.T).reshape(i1 - i0, L["h"], n) / math.sqrt(dh + L["dr"])
            hidden = torch.arange(n, device="cuda")[None, :] - (n - k) > torch.arange(i0, i1, device="cuda")[:, None]
            sc.masked_fill_(hidden[:, None, :], -math.inf)
            o = (torch.softmax(sc, 2).reshape(-1, n) @ key[:, :dc]).reshape(i1 - i0, L["h"], dc)
            out[cu[b] + i0:cu[b] + i1] = torch.stack([o[:, h] @ w_uv[h].T for h in range(L["h"])], 1)
    return out


EXACT = dict(rope=_exact_rope, write=_exact_write, read=_exact_read, attend=_exact_attend)


def exact(case, seed):
    return EXACT[case["kind"]](prepare(case, seed))
