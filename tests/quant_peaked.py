"""Attention over the 8-bit cache where single keys decide: weights that select, keys of large scores at the borders of
tiles, and a bound that follows the roundings one by one.  In NumPy; nothing here needs a GPU.

W_UK and W_UV hold one 1 in each latent column and each output row, so that q_lat and the up-projection are exact and an
output is one latent value of the merged row.  Bound of that output, o = sum p c~ over the keys that the row attends to:
  each probability rounds to fp16 once: half a step of 2^-11 of it, and no less than 2^-25 where fp16 is subnormal (the
    row's largest is at least 1 in the kernel's units, and so is their sum l, in which p is divided):
      2^-11 sum p |c~| + 2^-25 sum |c~| / l
  scores: sums of d_c + d_r fp32 products, each addition off by at most 2^-24 of sum |q k|, the scale's product and the
    exponential by 2^-21 together; a weight moves by that, relatively, and so does their sum:  2 e sum p |c~|
  sums over keys, the merge and the merged row's two bf16 halves: 2^-15 sum p |c~|
  the output: half a step of bf16, 2^-8 |o|."""
import math

import numpy as np
import torch

from quant_oracle import TABLE, e4m3, row_exponent

LOG2E = 1.4426950408889634
STEP = 8.5  # log2 units from one height to the next: more than the 8 that a running maximum may lag


def encode(c):
    """(codes, scales) of rows of finite values, by the format's definition."""
    e = row_exponent(c)
    value = e4m3(c * 2.0 ** -e[:, None].astype(np.float64))
    code = np.searchsorted(TABLE[:127], np.abs(value)).astype(np.uint8) | np.where(np.signbit(value), 128, 0).astype(np.uint8)
    return code, (e + 127).astype(np.uint8)


def decode(code, scale):
    return TABLE[code] * 2.0 ** (scale.astype(np.float64) - 127)[:, None]


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


class Peaked:
    """Sequences of `lens` cached tokens, the last `new` of each new ones.  Every 32 tokens the first and the last are
    keys of large scores for some rows: of heights 1 to 3, STEP apart.
      peaks "rope":   the score is the RoPE key's; each peak is seen by every other row of one wave (rows `per_wave` apart,
                      four waves).  Lower peaks hold larger values, so that each height counts in the output.
      peaks "latent": the score is the latent's; each peak is seen by one row of four."""

    def __init__(self, seed, h, dh, dv, dc, dr, new, lens, peaks, per_wave):
        r = np.random.default_rng(seed)
        self.h, self.dh, self.dv, self.dc, self.dr, self.new, self.lens = h, dh, dv, dc, dr, new, lens
        self.tau = 1 / math.sqrt(dh + dr)
        hh, cc, vv = np.arange(h), np.arange(dc), np.arange(dv)
        self.w_uk, self.w_uv = np.zeros((h, dh, dc)), np.zeros((h, dv, dc))
        self.pick_q = (cc[None] + hh[:, None]) % dh         # q_lat[h, c] = q[pick_q]
        self.pick_v = (vv[None] + dv * hh[:, None]) % dc    # out[h, v] = o[pick_v]
        self.w_uk[hh[:, None], self.pick_q, cc[None]] = 1
        self.w_uv[hh[:, None], vv[None], self.pick_v] = 1
        self.q, self.lat, self.rope = [], [], []
        for n, length in zip(new, lens):
            rows = n * h
            wave = np.arange(rows) // per_wave % 4
            peak = np.array([j for j in range(length - n) if j % 32 in (0, 31)], dtype=np.int64)
            owner, height = r.integers(0, 4, len(peak)), r.choice([1, 2, 3], len(peak), p=[1 / 6, 1 / 3, 1 / 2])
            q = np.zeros((rows, dh + dr))
            lat, rope = r.normal(size=(length, dc)), r.normal(size=(length, dr))
            if peaks == "rope":
                gain = 8.0
                q[:, dh:] = 0.5 * r.normal(size=(rows, dr))
                q[:, dh: dh + 4] = 0
                q[np.arange(rows), dh + wave] = np.where(np.arange(rows) % 2 == 0, gain, -gain)
                rope[:, :4] = 0
                rope[peak, owner] = height * STEP / (gain * self.tau * LOG2E)
                lat *= 2.0 ** -7
                lat[peak] *= (2.0 ** (STEP * (3 - height)))[:, None]
            else:
                q = r.normal(size=(rows, dh + dr))
                row = (owner * per_wave + per_wave // 2 - 1) % rows
                mine = bf16(q[row])[:, :dh][np.arange(len(peak))[:, None], self.pick_q[row % h]]
                lat[peak] = mine * (height * STEP / (self.tau * LOG2E * (mine ** 2).sum(1)))[:, None]
            self.q.append(bf16(q).reshape(n, h, dh + dr))
            self.lat.append(lat)
            self.rope.append(bf16(rope))
        cached = [encode(x) for x in self.lat]
        self.codes, self.scales = [c for c, _ in cached], [s for _, s in cached]
        self.lat = [decode(c, s) for c, s in cached]

    def attend(self, change=None):
        """(out, bound) of the packed new tokens; `change(b, keys, weights)` may alter what is summed."""
        out, bound = [], []
        for b, (n, length) in enumerate(zip(self.new, self.lens)):
            q, lat = self.q[b], self.lat[b]
            ql = np.take_along_axis(q, np.broadcast_to(self.pick_q, (n, self.h, self.dc)), 2).astype(np.float16).astype(np.float64)
            qq = np.concatenate([ql, q[:, :, self.dh:]], 2).reshape(n * self.h, -1) * self.tau
            k = np.concatenate([lat, self.rope[b]], 1)
            s = qq @ k.T
            e = (self.dc + self.dr) * 2.0 ** -24 * (np.abs(qq) @ np.abs(k).T).max(1, keepdims=True) + 2.0 ** -21 * (1 + np.abs(s).max(1, keepdims=True))
            token = np.arange(n * self.h)[:, None] // self.h
            s = np.where(np.arange(length)[None] < length - n + token + 1, s, -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            l = p.sum(1, keepdims=True)
            p /= l
            if change is not None:
                lat, p = change(b, lat.copy(), p.copy())
            o, size = p @ lat, p @ np.abs(lat)
            limit = (2.0 ** -11 + 2 * e + 2.0 ** -15) * size + 2.0 ** -25 * np.abs(lat).sum(0)[None] / l + 2.0 ** -8 * np.abs(o)
            pick = np.tile(self.pick_v, (n, 1))
            out.append(np.take_along_axis(o, pick, 1).reshape(n, self.h, self.dv))
            bound.append(np.take_along_axis(limit, pick, 1).reshape(n, self.h, self.dv))
        return np.concatenate(out), np.concatenate(bound)
