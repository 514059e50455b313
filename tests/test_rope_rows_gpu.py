"""eg_mla_rope_rows against its formula in 64 bits: both layouts, parts of rows of any size and alignment, strides, far
positions, stretched contexts, the way back."""
import math

import numpy as np
import pytest
import torch

from paper_2509_16686_amd import binding as B
from quant_oracle import BF, HALF_STEP, I32, frequencies, rotate

pytestmark = pytest.mark.gpu

# A rotated value errs by its rounding, half a step of itself, and by the angle's, 2^-26 turns (2 pi 2^-26 < 2^-23 rad)
# and a little, fp32 sines and products (a few 2^-24) of the pair's magnitude: below 2^-20 of it together.
ANGLE = 2.0 ** -20


def check(got, x, off, rd, positions, f, half, magnitude=1.0, inverse=False, copied=True):
    want = x.double().cpu().numpy().copy()
    part = want[..., off:off + rd].copy()
    want[..., off:off + rd] = rotate(part, positions.cpu().numpy(), f, half, magnitude, inverse)
    a, b = (part[..., : rd // 2], part[..., rd // 2:]) if half else (part[..., 0::2], part[..., 1::2])
    r = np.hypot(a, b) * magnitude
    size = np.concatenate([r, r], -1) if half else np.repeat(r, 2, -1)
    got = got.double().cpu().numpy()
    bound = HALF_STEP[x.dtype] * np.abs(want)
    bound[..., off:off + rd] += ANGLE * size
    assert (np.abs(got - want) <= bound).all()


def rows(seed, shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("n,h,dim,off,rd", [
    (1, 1, 64, 0, 64), (8, 16, 192, 128, 64), (5, 5, 64, 40, 24), (3, 12, 128, 0, 128), (2, 3, 90, 7, 18), (4, 1, 2, 0, 2),
    (3, 2, 66, 1, 62), (7, 4, 80, 16, 64), (1, 130, 192, 128, 64), (2, 2, 700, 60, 640), (300, 16, 72, 8, 64), (1, 3, 11, 4, 0),
    (600, 128, 40, 8, 32),
])
def test_against_the_formula(gpu, half, dtype, n, h, dim, off, rd):
    x = rows(n + dim, (n, h, dim), dtype)
    positions = torch.randint(0, 1 << 20, (n,), device="cuda", dtype=I32)
    out = torch.full_like(x, 7.0)
    B.rope_rows(B.make_rope(layout=int(half)), x, positions, out, rope_dim=rd, rope_offset=off)
    check(out, x, off, rd, positions, frequencies(max(rd, 2)) if rd else np.zeros(0), half)


@pytest.mark.parametrize("half", [False, True])
def test_far_and_negative_positions(gpu, half):
    x = rows(1, (8, 2, 96), BF)
    positions = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6, 123456789, 4097], device="cuda", dtype=I32)
    out = torch.empty_like(x)
    B.rope_rows(B.make_rope(layout=int(half), theta=1e6), x, positions, out, rope_dim=64)
    # (the angles of the oracle, position times frequency in 64 bits, are themselves off by 2^31 2^-53)
    check(out, x, 32, 64, positions, frequencies(64, 1e6), half)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("factor,trained", [(4.0, 4096), (40.0, 2048), (8.0, 0)])
def test_stretched_context(gpu, half, factor, trained):
    f = B.rope_frequencies(64, factor, trained)
    want = frequencies(64, factor=factor, trained=trained)
    assert np.allclose(f, want, rtol=1e-12, atol=0)
    x = rows(2, (9, 4, 192), BF)
    positions = torch.arange(9, device="cuda", dtype=I32) * 12345
    out = torch.empty_like(x)
    m = 0.1 * math.log(factor) + 1
    B.rope_rows(B.make_rope(layout=int(half), frequencies=f, magnitude=m), x, positions, out, rope_dim=64)
    check(out, x, 128, 64, positions, want, half, np.float64(np.float32(m)))


def test_given_frequencies(gpu):
    f = [0.0, -0.5, 7.25, 6.283185307179586, 64.0, -1e-12, -64.0, 1e-3]
    x = rows(3, (6, 3, 16), torch.float32)
    positions = torch.tensor([0, 1, 2, 3, 50, 7], device="cuda", dtype=I32)
    out = torch.empty_like(x)
    B.rope_rows(B.make_rope(frequencies=f), x, positions, out, rope_dim=16)
    check(out, x, 0, 16, positions, np.array(f), False)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_in_place_and_back(gpu, half, dtype):
    x = rows(4, (33, 6, 100), dtype)
    positions = torch.randint(0, 100000, (33,), device="cuda", dtype=I32)
    rope, y = B.make_rope(layout=int(half)), x.clone()
    B.rope_rows(rope, y, positions, y, rope_dim=48, rope_offset=20)
    apart = torch.empty_like(x)
    B.rope_rows(rope, x, positions, apart, rope_dim=48, rope_offset=20)
    assert torch.equal(y, apart)
    z = torch.empty_like(y)
    B.rope_rows(rope, y, positions, z, rope_dim=48, rope_offset=20, inverse=True)
    check(z, y, 20, 48, positions, frequencies(48), half, inverse=True)
    # there and back: a value is rounded twice, and each of a pair takes part of the other's rounding
    size = x.double().abs().amax()
    assert (z.double() - x.double()).abs().max() <= 4 * HALF_STEP[dtype] * size + 2 * ANGLE * size


@pytest.mark.parametrize("half", [False, True])
def test_gradient(gpu, half):
    """inverse is the gradient: <g, R(x + d)> - <g, R(x - d)> = 2 <R^T g, d>."""
    positions = torch.tensor([3, 70000], device="cuda", dtype=I32)
    x, g, d = (rows(s, (2, 3, 40), torch.float32) for s in (5, 6, 7))
    rope = B.make_rope(layout=int(half), frequencies=B.rope_frequencies(24, 4.0, 1000), magnitude=1.25)
    turn = lambda t, **kw: (lambda o: (B.rope_rows(rope, t, positions, o, rope_dim=24, rope_offset=8, **kw), o.double())[1])(torch.empty_like(t))
    back = turn(g, inverse=True)
    step = 0.5 * d
    left = (g.double() * (turn(x + step) - turn(x - step))).sum()
    right = 2 * (back * step.double()).sum()
    # (x + step is rounded in fp32: a few 2^-24 of 240 terms of magnitude about one)
    assert abs(float(left - right)) <= 240 * 16 * 2.0 ** -24
    check(back.float(), g, 8, 24, positions, frequencies(24, factor=4.0, trained=1000), half, 1.25, inverse=True)


def test_strides(gpu):
    big = rows(8, (6, 1000), BF)
    positions = torch.randint(0, 5000, (6,), device="cuda", dtype=I32)
    f = frequencies(64)
    for x in (big[:, 8:8 + 4 * 96].unflatten(1, (4, 96)), big[:, 3:3 + 4 * 96].unflatten(1, (4, 96)),
              big.as_strided((6, 4, 96), (1000, 200, 1)), big.as_strided((6, 4, 96), (0, 200, 1)),
              big.as_strided((6, 4, 96), (1000, 0, 1)), rows(9, (4, 6, 96), BF).transpose(0, 1)):
        for half in (False, True):
            out = torch.empty((6, 4, 96), dtype=BF, device="cuda")
            B.rope_rows(B.make_rope(layout=int(half)), x, positions, out, rope_dim=64)
            check(out, x, 32, 64, positions, f, half)
            room = torch.full((4, 7, 104), 5.0, dtype=BF, device="cuda")
            B.rope_rows(B.make_rope(layout=int(half)), x, positions, room[:, :6, 3:99].transpose(0, 1), rope_dim=64)
            assert torch.equal(room[:, :6, 3:99].transpose(0, 1), out)
            assert bool((room[:, 6] == 5).all()) and bool((room[:, :, :3] == 5).all()) and bool((room[:, :, 99:] == 5).all())


def test_not_finite_values_stay_with_their_pair(gpu):
    x = rows(10, (2, 2, 64), BF)
    x[0, 1, 5], x[1, 0, 40], x[1, 1, 0] = math.inf, math.nan, -math.inf
    out = torch.empty_like(x)
    B.rope_rows(B.make_rope(), x, torch.tensor([5, 9], device="cuda", dtype=I32), out, rope_dim=64)
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    for i, h, m in ((0, 1, 2), (1, 0, 20), (1, 1, 0)):
        want[i, h, 2 * m: 2 * m + 2] = True
    assert torch.equal(bad, want)


def test_more_work_groups_than_one_dimension_takes(gpu):
    n = (1 << 24) + 1001
    x = rows(11, (n, 1, 8), BF)
    positions = torch.arange(n, device="cuda", dtype=I32)
    out = torch.empty_like(x)
    B.rope_rows(B.make_rope(), x, positions, out, rope_dim=4)
    at = torch.tensor([0, 1, 12345, (1 << 20) - 1, 1 << 20, (1 << 24) - 1, 1 << 24, n - 2, n - 1], device="cuda")
    check(out[at], x[at], 4, 4, positions[at], frequencies(4), False)
    B.rope_rows(B.make_rope(), out, positions, out, rope_dim=4, inverse=True)
    # there and back, a value is rounded twice, and each of a pair takes part of the other's rounding
    assert (out.float() - x.float()).abs().max() <= 4 * 2.0 ** -8 * x.float().abs().max()
