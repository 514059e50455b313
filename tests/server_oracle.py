"""Plain 64-bit forms of the operators around the decode (page tables, query and key rows, shared prefix, page means,
scores and selection), in NumPy and one sequence after the other, and the seeded layers that their tests run on."""
import numpy as np
import torch

from paper_2509_16686_amd import binding as B

I32 = torch.int32


def ceil_div(a, b):
    return -(-a // b)


def page_plan(page, cached, new, base, table, free, count, max_tokens):
    """(table, lens, cu, positions, slots, count) of eg_mla_page_plan; int64 NumPy arrays in and out."""
    table = table.copy()
    nb, width = table.shape
    cap, count = width * page, min(max(count, 0), len(free))
    cached = np.clip(cached, 0, cap)
    new = np.maximum(new, 0)
    lens, cu = cached.copy(), np.zeros(nb + 1, dtype=np.int64)
    positions, slots = np.zeros(max_tokens, dtype=np.int64), np.full(max_tokens, -1, dtype=np.int64)
    tokens = pages = taken = 0
    for b in range(nb):
        tokens += int(new[b])
        cu[b + 1] = min(tokens, max_tokens)
        n = cu[b + 1] - cu[b]
        at = cached[b] + np.arange(n)
        positions[cu[b]:cu[b + 1]] = (0 if base is None else base[b]) + at
        have, want = ceil_div(int(cached[b]), page), ceil_div(int(cached[b] + new[b]), page)
        if cached[b] + new[b] > cap:
            continue
        pages += want - have
        if tokens > max_tokens or (want > have and pages > count):
            continue
        for p in range(have, want):
            table[b, p] = free[count - 1 - taken]
            taken += 1
        lens[b] = cached[b] + new[b]
        pg = table[b, at // page] if n else np.zeros(0, dtype=np.int64)
        ok = (pg >= 0) & (pg < (2 ** 31 - 1) // page)
        slots[cu[b]:cu[b + 1]] = np.where(ok, pg * page + at % page, -1)
    return table, lens, cu, positions, slots, count - taken


def page_release(page, lens, ended, table, free, count):
    """(free, lens, count) of eg_mla_page_release."""
    free, lens = free.copy(), lens.copy()
    count = min(max(count, 0), len(free))
    for b in np.flatnonzero(ended):
        for p in table[b, : ceil_div(int(min(max(lens[b], 0), table.shape[1] * page)), page)]:
            if count < len(free):
                free[count] = p
                count += 1
        lens[b] = 0
    return free, lens, count


def norm(x, w):
    return x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6) * w


def rope(x, positions, theta=10000.0):
    """Rotation of adjacent pairs of the last dim, x [n, ..., d]."""
    d = x.shape[-1]
    if d == 0:
        return x
    freq = np.asarray(theta, dtype=np.longdouble) ** (np.arange(0, d, 2, dtype=np.longdouble) / -d)
    angle = np.asarray(positions, dtype=np.longdouble)[:, None] * freq
    angle = angle.reshape((x.shape[0],) + (1,) * (x.ndim - 2) + (d // 2,))
    cs, sn = np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64)
    out = np.empty_like(x)
    out[..., 0::2] = x[..., 0::2] * cs - x[..., 1::2] * sn
    out[..., 1::2] = x[..., 0::2] * sn + x[..., 1::2] * cs
    return out


class Layer:
    """A seeded layer with a paged cache on the GPU, and the same values in 64 bits."""

    def __init__(self, *, h, dh, dv, dc, dr, dtype, page, pages, vocab=211, seed=0, scale=0.0):
        self.h, self.dh, self.dv, self.dc, self.dr, self.page, self.pages = h, dh, dv, dc, dr, page, pages
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.storage = dtype
        self.g = torch.Generator().manual_seed(seed)
        self.tau = scale if scale > 0 else 1.0 / np.sqrt(dh + dr)
        self.dims = B.make_dims(num_heads=h, head_dim=dh, v_head_dim=dv, latent_dim=dc, rope_dim=dr, vocab_size=vocab,
                                page_size=page, softmax_scale=scale, dtype=B.BF16 if dtype == "bf16" else B.FP32)
        unit = 1.0 if dtype == "bf16" else 1 / np.sqrt(dc)  # the fp32 bar is absolute: outputs below one
        self.cache = self.normal((pages * page, dc + dr), unit)
        self.gate = self.normal((vocab, dc), 0.1, 1.0)
        self.w_uk, self.w_uv = self.normal((h, dh, dc), 1 / np.sqrt(dc)), self.normal((h, dv, dc), 1 / np.sqrt(dc))
        self.ids = self.ints(vocab, pages * page)

    def normal(self, shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=self.g) * std + mean).to(self.dtype).cuda()

    def ints(self, hi, n):
        return torch.randint(0, hi, (n,), generator=self.g, dtype=I32).cuda()

    def query(self, b, factor=1.0):
        unit = factor if self.storage == "bf16" else factor / np.sqrt(self.dh)
        return self.normal((b, self.h, self.dh + self.dr), unit)

    def table(self, lens, width=None, spare=0):
        """A page table with random pages, -1 behind each sequence's; `spare` pages that no sequence holds."""
        per = [ceil_div(n, self.page) for n in lens]
        order = torch.randperm(self.pages, generator=self.g).to(I32)
        assert sum(per) + spare <= self.pages
        t = torch.full((len(lens), max(width or 0, max(per + [1]))), -1, dtype=I32)
        at = 0
        for b, n in enumerate(per):
            t[b, :n] = order[at:at + n]
            at += n
        return t.cuda(), order[at:at + spare].cuda()

    def f64(self, t):
        return t.detach().to(torch.float64).cpu().numpy()

    def rows(self, pages, n):
        """[c (.) G[id] | k^R] of the first n tokens of a list of pages."""
        at = (np.asarray([int(p) for p in pages], dtype=np.int64)[:, None] * self.page + np.arange(self.page)).reshape(-1)[:n]
        x = self.f64(self.cache[torch.from_numpy(at).cuda()])
        ids = self.ids.cpu().numpy()[at].clip(0, self.gate.shape[0] - 1)
        x[:, : self.dc] *= self.f64(self.gate)[ids]
        return x

    def absorbed(self, q):
        """[W_UK^T q^C | q^R] of query rows [B, H, d_h + d_r]."""
        ql = np.einsum("bhd,hdc->bhc", q[..., : self.dh], self.f64(self.w_uk))
        return np.concatenate([ql, q[..., self.dh:]], -1)

    def attend(self, q, rows_of):
        """out[b] = W_UV softmax(tau q . rows) rows over the rows rows_of(b) of each sequence; no rows give zeros."""
        qf = self.absorbed(self.f64(q))
        out = np.zeros((q.shape[0], self.h, self.dv))
        w = self.f64(self.w_uv)
        for b in range(q.shape[0]):
            rows = rows_of(b)
            if len(rows):
                s = self.tau * qf[b] @ rows.T
                p = np.exp(s - s.max(1, keepdims=True))
                o = (p / p.sum(1, keepdims=True)) @ rows[:, : self.dc]
                out[b] = np.einsum("hc,hvc->hv", o, w)
        return out


def select(scores, lens, page, keep, keep_first, keep_last):
    """Chosen columns of each sequence (lists in order) and their tokens."""
    cols, tokens = [], []
    for s, n in zip(scores, lens):
        have = ceil_div(int(n), page)
        always = [j for j in range(have) if j < keep_first or j >= have - keep_last]
        if have > keep:
            value = np.where(np.isnan(s), -np.inf, s)
            others = sorted((j for j in range(have) if j not in always), key=lambda j: (-value[j], j))
            chosen = sorted(always + others[: keep - len(always)])
        else:
            chosen = list(range(have))
        cols.append(chosen)
        tokens.append(int(n) - (have - len(chosen)) * page)
    return cols, tokens
