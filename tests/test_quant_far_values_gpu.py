"""Rows of the 8-bit cache with values past fp16's range, or codes that are NaN: new tokens that do not attend to such a
row do not notice it, the others get NaN; the largest values that fp16 holds stay values."""
import numpy as np
import pytest
import torch

from paper_2509_16686_amd import binding as B
from quant_oracle import BF, U8, Layer, check_attend, offsets

pytestmark = pytest.mark.gpu

WIDE = 1 << 20  # tokens of capacity: enough for blocks of 128 rows wherever there are 48 rows a sequence
SHAPES = {"odd": (5, 40, 56, 48, 24), "no_rope": (16, 64, 64, 64, 0), "h16": (16, 128, 128, 128, 64), "d144": (16, 64, 136, 144, 64),
          "mla320": (16, 128, 128, 320, 64), "h128": (128, 128, 128, 512, 64), "d496": (3, 24, 24, 496, 16)}
LENS, NEW = [70, 37, 160], [20, 1, 33]


def layer(shape, wide):
    L = Layer(50, *SHAPES[shape], page=16, rows=16 * 24)
    table = L.table(LENS, WIDE // 16 if wide else None)
    return L, table, L.slots_of(table), L.normal((sum(NEW), L.h, L.dh + L.dr))


def put(L, slot, values):
    """A row of the layer's cache with `values` as its gated latent, by eg_mla_quant_write."""
    kv = torch.cat([values.to(BF), L.normal((L.dr,))])[None].contiguous()
    B.quant_write(L.dims, None, kv, None, torch.tensor([slot], dtype=torch.int32, device="cuda"), L.codes, L.scales)


def far(L, slot, kind):
    """The row becomes one whose values fp16 does not hold, in one place or in all."""
    x = L.normal((L.dc,))
    if kind == "nan code":       # which no call writes
        L.codes[slot, 7] = 0x7F
    elif kind == "-nan code":
        L.codes[slot, L.dc - 1] = 0xFF
    elif kind == "all nan":      # memory that no call has written
        L.codes[slot], L.scales[slot] = 0xFF, 0xFF
    elif kind == "1e5":
        x[L.dc // 2] = 1e5
        put(L, slot, x)
    elif kind == "-66000":
        x[0] = -66000.0
        put(L, slot, x)
    else:
        put(L, slot, x * 1e30)


@pytest.mark.parametrize("wide", [0, WIDE])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("kind", ["nan code", "-nan code", "all nan", "1e5", "-66000", "1e30"])
def test_tokens_that_are_not_attended_to(gpu, kind, shape, wide):
    """One of the new tokens' rows, and the last of a decode: those before give the same bits whatever it holds."""
    L, table, at, q = layer(shape, wide)
    first = np.cumsum([0] + NEW)
    plain = L.run(q, offsets(NEW), LENS, table)
    seen = torch.zeros(sum(NEW), dtype=torch.bool, device="cuda")
    for b, i in ((0, 13), (1, 0), (2, 32)):  # new token i of sequence b: seen by it and those behind it
        far(L, int(at(b, LENS[b])[LENS[b] - NEW[b] + i]), kind)
        seen[first[b] + i: first[b + 1]] = True
    out = L.run(q, offsets(NEW), LENS, table)
    assert torch.equal(out[~seen], plain[~seen])
    assert bool(torch.isnan(out[seen]).all())


@pytest.mark.parametrize("wide", [0, WIDE])
@pytest.mark.parametrize("shape", ["h16", "mla320", "h128"])
def test_the_largest_values_of_fp16(gpu, shape, wide):
    """Up to 61440, the largest that a code and a power of two make below 65504, in rows of scale 2^7 and 2^8."""
    L, table, at, q = layer(shape, wide)
    for b, j, top in ((0, 3, 57344.0), (1, 36, 61440.0), (2, 130, -61440.0), (2, 159, 63000.0)):
        x = L.normal((L.dc,))
        x[5] = top
        put(L, int(at(b, LENS[b])[j]), x)
    assert sorted(L.scales.unique().tolist())[-2:] == [134, 135]
    q[..., : L.dh] *= 2.0 ** -16  # scores stay of order one
    out = L.run(q, offsets(NEW), LENS, table)
    assert bool(torch.isfinite(out).all())
    check_attend(out, *L.oracle(q, NEW, LENS, at))
