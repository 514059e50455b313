"""The 8-bit cache written and read back (eg_mla_quant_write, eg_mla_quant_read) against 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from paper_2509_16686_amd import binding as B
from quant_oracle import (BF, HALF_STEP, I32, U8, Layer, cache_rows, e4m3, frequencies, ints, norm, offsets, rotate,
                          row_exponent)

pytestmark = pytest.mark.gpu

# A gated latent before its rounding errs by fp32 norms and products: the sum of squares of d_c <= 512 terms (its tree adds
# at most 2^-24 (8 + 6) and squares 2^-24), root, quotient and three products: below 2^-19 of itself.
LATENT = 2.0 ** -19


def want_rows(kv, dc, kv_w, k_w, gate, positions, rope):
    """(gated latents, RoPE keys) in 64 bits; rope: (frequencies, half, magnitude) or None."""
    f = lambda t: None if t is None else t.double().cpu().numpy()
    x = f(kv)
    c = norm(x[:, :dc], f(kv_w))
    if gate is not None:
        c = c * f(gate)
    k = norm(x[:, dc:], f(k_w))
    if rope is not None and k.shape[1]:
        k = rotate(k, positions.cpu().numpy(), *rope)
    return c, k


def check_rows(codes, scales, dc, c, k):
    """Cache rows against gated latents c and keys k."""
    got = cache_rows(codes, scales, dc)
    e = scales.cpu().numpy().astype(int) - 127
    # the exponent, where the largest magnitude is not within LATENT of a border
    top = np.abs(c).max(1)
    lo, hi = row_exponent(c * (1 - LATENT)), row_exponent(c * (1 + LATENT))
    assert ((e >= lo) & (e <= hi)).all()
    scale = 2.0 ** e[:, None].astype(np.float64)
    # the code of a value within LATENT of the exact one: rounding is monotonic
    a, b = e4m3(np.clip(np.abs(c) * (1 - LATENT) / scale, 0, 448)), e4m3(np.clip(np.abs(c) * (1 + LATENT) / scale, 0, 448))
    x = np.abs(got[:, :dc]) / scale
    assert ((x >= a) & (x <= b)).all()
    assert (np.sign(got[:, :dc]) * np.sign(c) >= 0).all()
    r = got[:, dc:]
    if r.shape[1]:
        pair = np.abs(k).max(1, keepdims=True) * 1.5  # the other value of a pair is at most the row's largest
        assert (np.abs(r - k) <= HALF_STEP[BF] * np.abs(k) + (2.0 ** -19) * pair).all()
    assert (top >= 0).all()


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("norms,gated", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("h,dc,dr,n", [(1, 16, 8, 1), (5, 48, 24, 7), (12, 64, 64, 40), (16, 128, 64, 33), (16, 144, 0, 5),
                                       (2, 256, 32, 70), (16, 320, 64, 9), (4, 512, 64, 130), (4, 512, 2 * 8, 17)])
def test_write(gpu, half, norms, gated, h, dc, dr, n):
    L = Layer(1, h, 64, 64, dc, dr, rows=256)
    kv = L.normal((n, dc + dr), 2.0)
    kv_w = L.normal((dc,), 0.2, 1.0) if norms else None
    k_w = L.normal((dr,), 0.2, 1.0) if norms else None
    ids, positions, slots = L.ints(300, n), L.ints(1 << 17, n), L.perm(256)[:n].contiguous()
    before = L.codes.clone(), L.scales.clone()
    B.quant_write(L.dims, B.make_rope(layout=int(half)), kv, positions, slots, L.codes, L.scales,
                  gate_table=L.gate if gated else None, token_ids=ids if gated else None, kv_norm_w=kv_w,
                  k_norm_w=k_w if dr else None)
    at = slots.long()
    c, k = want_rows(kv, dc, kv_w, k_w, L.gate[ids.long()] if gated else None, positions, (frequencies(max(dr, 2)), half))
    check_rows(L.codes[at], L.scales[at], dc, c, k)
    rest = torch.ones(256, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(L.codes[rest], before[0][rest]) and torch.equal(L.scales[rest], before[1][rest])


def test_write_of_given_rows_is_exact(gpu):
    """Without norms, gate and rotation: values on the grid keep themselves, ties go to the even code, borders hold."""
    L = Layer(2, 4, 64, 64, 128, 64, rows=64)
    kv = torch.zeros((12, 192), dtype=BF, device="cuda")
    kv[0, :4] = torch.tensor([448.0, -448.0, 17.0, 19.0])         # ties: 17 -> 16, 19 -> 20
    kv[1, :3] = torch.tensor([450.0, 1.0, -3.0])                  # past 448: the next power of two
    kv[2, :2] = torch.tensor([2.0 ** -100, -(2.0 ** -101)])
    kv[3, :2] = torch.tensor([2.0 ** -126, 2.0 ** -130])          # the least exponents
    kv[4, :2] = torch.tensor([3.0e38, -1.0])                      # the greatest
    kv[5, :4] = torch.tensor([448.0, 2.0 ** -6, 2.0 ** -9, 2.0 ** -10])  # subnormal codes; half of the least: to zero
    kv[6, :4] = torch.tensor([224.0, 448.0, 3 * 2.0 ** -10, -5 * 2.0 ** -10])  # halves between subnormals
    kv[8, 127] = -0.0
    kv[9, :128] = torch.arange(128) - 64.0
    kv[10, :128], kv[11, :128] = L.normal((128,)), L.normal((128,), 1e-3)
    kv[:, 128:] = L.normal((12, 64))
    slots = ints(range(20, 32))
    B.quant_write(L.dims, None, kv, None, slots, L.codes, L.scales)
    x = kv.double().cpu().numpy()
    e = row_exponent(x[:, :128])
    assert np.array_equal(L.scales[20:32].cpu().numpy().astype(int) - 127, e)
    want = e4m3(x[:, :128] * 2.0 ** -e[:, None].astype(np.float64)) * 2.0 ** e[:, None].astype(np.float64)
    got = cache_rows(L.codes[20:32], L.scales[20:32], 128)
    assert np.array_equal(got[:, :128], want) and np.array_equal(got[:, 128:], x[:, 128:])
    # a second quantisation of the values changes nothing
    out = torch.empty((12, 192), dtype=BF, device="cuda")
    cu, table = ints([0, 12]), ints([[1]][0]).reshape(1, 1)
    B.quant_read(L.dims, L.codes, L.scales, ints([4]), cu, table, out)
    codes, scales = L.codes.clone(), L.scales.clone()
    B.quant_write(L.dims, None, out, None, slots, codes, scales)
    keep = torch.ones(64, dtype=torch.bool)
    keep[23] = False  # (2^-130 of row 3 is code zero, and 2^-126 needs no more than its own exponent)
    assert np.array_equal(cache_rows(codes, scales, 128)[keep], cache_rows(L.codes, L.scales, 128)[keep])


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("norms", [False, True])
def test_not_finite_latents(gpu, bad, norms):
    L = Layer(3, 4, 64, 64, 64, 64, rows=64)
    kv = L.normal((4, 128))
    kv[1, 63], kv[3, 64 + 5] = bad, bad
    w = (L.normal((64,), 0.1, 1.0), L.normal((64,), 0.1, 1.0)) if norms else (None, None)
    B.quant_write(L.dims, B.make_rope(), kv, ints([1, 2, 3, 4]), ints([0, 1, 2, 3]), L.codes, L.scales, kv_norm_w=w[0], k_norm_w=w[1])
    assert (L.scales[:4] == 255).tolist() == [False, True, False, False]
    assert bool((L.codes[1, :64] == 0).all())
    out = torch.empty((4, 128), dtype=BF, device="cuda")
    B.quant_read(L.dims, L.codes, L.scales, None, ints([0, 4]), ints([0]).reshape(1, 1), out)
    nan = torch.isnan(out[:, :64])
    assert bool(nan[1].all()) and not bool(nan[[0, 2, 3]].any())
    assert bool((~torch.isfinite(out[3, 64:])).any()) and bool(torch.isfinite(out[:3, 64:]).all())


def test_infinite_gate_and_overflow(gpu):
    L = Layer(4, 4, 64, 64, 64, 0, rows=64)
    L.gate[7, 3], L.gate[8, :] = math.inf, 3e38
    kv = torch.full((3, 64), 100.0, dtype=BF, device="cuda")
    B.quant_write(L.dims, None, kv, None, ints([0, 1, 2]), L.codes, L.scales, gate_table=L.gate, token_ids=ints([7, 8, 9]))
    assert (L.scales[:3] == 255).tolist() == [True, True, False]


def test_skipped_slots_clamped_ids_and_strides(gpu):
    L = Layer(5, 4, 64, 64, 96, 32, rows=64)
    wide = L.normal((8, 96 + 32 + 72))
    kv = wide[:, 40:168]
    ids = ints([-5, 300, 10 ** 9, 5, 6, 7, 8, 9])
    slots = ints([3, 60, 63, -1, 64, 2 ** 31 - 1, -2 ** 31, 0])
    before = L.codes.clone(), L.scales.clone()
    positions = ints(range(8))
    B.quant_write(L.dims, B.make_rope(), kv, positions, slots, L.codes, L.scales, gate_table=L.gate, token_ids=ids)
    done, at = [0, 1, 2, 7], [3, 60, 63, 0]
    c, k = want_rows(kv, 96, None, None, L.gate[ids.long().clamp(0, 299)], positions, (frequencies(32), False))
    check_rows(L.codes[at], L.scales[at], 96, c[done], k[done])
    rest = [i for i in range(64) if i not in at]
    assert torch.equal(L.codes[rest], before[0][rest]) and torch.equal(L.scales[rest], before[1][rest])


def test_write_magnitude_and_frequencies(gpu):
    L = Layer(6, 4, 64, 64, 128, 64, rows=64)
    kv, positions = L.normal((6, 192)), ints([0, 1, 99, 4096, 40000, 2 ** 31 - 1])
    for half in (False, True):
        rope = B.make_rope(layout=int(half), frequencies=B.rope_frequencies(64, 16.0, 4096), magnitude=1.25)
        B.quant_write(L.dims, rope, kv, positions, ints(range(6)), L.codes, L.scales)
        c, k = want_rows(kv, 128, None, None, None, positions, (frequencies(64, factor=16.0, trained=4096), half, 1.25))
        check_rows(L.codes[:6], L.scales[:6], 128, c, k)


def test_write_agrees_with_the_bf16_cache(gpu):
    """The keys' rotation is the one of eg_mla_qk_norm_rope, bit for bit."""
    L = Layer(7, 4, 64, 64, 128, 64, rows=64)
    kv, positions, slots = L.normal((9, 192)), L.ints(1 << 20, 9), L.perm(64)[:9].contiguous()
    ids, w, kw = L.ints(300, 9), L.normal((128,), 0.1, 1.0), L.normal((64,), 0.1, 1.0)
    cache, id_cache = torch.zeros((64, 192), dtype=BF, device="cuda"), torch.zeros(64, dtype=I32, device="cuda")
    B.qk_norm_rope(L.dims, None, None, kv, cache, id_cache, ids, positions, slots, kv_norm_w=w, k_norm_w=kw)
    B.quant_write(L.dims, B.make_rope(), kv, positions, slots, L.codes, L.scales, gate_table=L.gate, token_ids=ids,
                  kv_norm_w=w, k_norm_w=kw)
    a, b = L.codes[slots.long(), 128:].contiguous().view(BF).double(), cache[slots.long(), 128:].double()
    assert (a - b).abs().max() <= 2.0 ** -7 * b.abs().max()  # one rounding apart at most
    assert (a == b).double().mean() > 0.99


@pytest.mark.parametrize("paged", [True, False])
@pytest.mark.parametrize("dc,dr,page", [(16, 8, 1), (48, 24, 24), (128, 64, 16), (320, 64, 64), (512, 0, 7), (512, 64, 16)])
def test_read(gpu, paged, dc, dr, page):
    lens = [0, 1, 37, 64, 5, 0]
    L = Layer(8, 4, 64, 64, dc, dr, page=page, rows=page * (6 * -(-64 // page)))
    width = -(-64 // page)
    table = L.table(lens, width) if paged else None
    first = [0, 0, 5, 16, 4, 0]
    new = [n - f for n, f in zip(lens, first)]
    total = sum(new)
    out = torch.full((total + 9, dc + dr), 5.0, dtype=BF, device="cuda")
    rows = cache_rows(L.codes, L.scales, dc)
    B.quant_read(L.dims, L.codes, L.scales, ints(first), offsets(new), table, out, max_pages_per_seq=width)
    at = L.slots_of(table) if paged else lambda b, n: b * width * page + np.arange(n)
    want = np.concatenate([rows[at(b, n)][f:] for b, (n, f) in enumerate(zip(lens, first))])
    assert np.array_equal(out[:total].double().cpu().numpy(), want)  # bf16 holds a code times its power of two
    assert bool((out[total:] == 5).all())
    if paged:
        again = torch.empty((sum(lens), dc + dr), dtype=BF, device="cuda")
        B.quant_read(L.dims, L.codes, L.scales, None, offsets(lens), table, again)
        assert np.array_equal(again.double().cpu().numpy(), np.concatenate([rows[at(b, n)] for b, n in enumerate(lens)]))


def test_read_many_sequences_and_bad_pages(gpu):
    L = Layer(9, 4, 64, 64, 64, 32, page=8, rows=4096)
    lens = [i % 3 for i in range(4096)]
    table = torch.randint(0, 512, (4096, 1), device="cuda", dtype=I32)
    table[5], table[8], table[2] = -3, 512, 2 ** 31 - 1
    out = torch.empty((sum(lens), 96), dtype=BF, device="cuda")
    B.quant_read(L.dims, L.codes, L.scales, None, offsets(lens), table, out)
    rows = cache_rows(L.codes, L.scales, 64)
    t = table.cpu().numpy()[:, 0].astype(np.int64).clip(0, 511)
    want = np.concatenate([rows[t[b] * 8 + np.arange(n)] for b, n in enumerate(lens)])
    assert np.array_equal(out.double().cpu().numpy(), want)


def test_read_past_the_capacity_and_offsets_out_of_order(gpu):
    L = Layer(10, 4, 64, 64, 64, 32, page=8, rows=64)
    rows = cache_rows(L.codes, L.scales, 64)
    table = ints([3, 1]).reshape(1, 2)
    out = torch.empty((20, 96), dtype=BF, device="cuda")
    B.quant_read(L.dims, L.codes, L.scales, ints([-4]), ints([0, 20]), table, out)
    j = np.minimum(np.arange(20), 15)
    assert np.array_equal(out.double().cpu().numpy(), rows[np.array([3, 1])[j // 8] * 8 + j % 8])
    for cu in ([0, 5, 2, 2 ** 31 - 1], [7, -5, 90, 3], [-2 ** 31, 2 ** 31 - 1, 0, 20]):  # not allowed; stays inside
        B.quant_read(L.dims, L.codes, L.scales, ints([2 ** 31 - 1, 1, 0]), ints(cu), torch.zeros((3, 2), dtype=I32, device="cuda"), out)
    torch.cuda.synchronize()
