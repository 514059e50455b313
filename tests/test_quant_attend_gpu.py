"""eg_mla_quant_attend against explicit attention over the same 8-bit rows in 64 bits: head counts, widths, lengths, new
tokens, page sizes, rows without tokens, rows that stand for NaN, workspaces, streams."""
import math

import numpy as np
import pytest
import torch

from paper_2509_16686_amd import binding as B
from quant_oracle import BF, I32, U8, Layer, cache_rows, check_attend, ints, offsets

pytestmark = pytest.mark.gpu

#         h   dh   dv   dc   dr
SHAPES = {"one": (1, 8, 8, 16, 0), "odd": (5, 40, 56, 48, 24), "kv64": (12, 64, 64, 64, 64), "h16": (16, 128, 128, 128, 64),
          "h20": (20, 128, 96, 128, 32), "d144": (16, 64, 136, 144, 64), "mla320": (16, 128, 128, 320, 64),
          "h24": (24, 128, 128, 512, 64), "h128": (128, 128, 128, 512, 64), "h130": (130, 16, 8, 64, 8), "d496": (3, 24, 24, 496, 16),
          "tall": (2, 1024, 1024, 64, 64)}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("page,lens", [(16, [1]), (64, [64, 0, 63, 65, 1]), (24, [200, 300, 7]), (1, [33, 2, 17, 16])])
def test_decode(gpu, shape, page, lens):
    L = Layer(len(lens), *SHAPES[shape], page=page, rows=page * (sum(-(-n // page) for n in lens) + 2))
    table = L.table(lens)
    q = L.normal((len(lens), L.h, L.dh + L.dr))
    check_attend(L.run(q, None, lens, table), *L.oracle(q, [1] * len(lens), lens, L.slots_of(table)))


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("new,lens", [([3], [3]), ([2, 0, 5, 1], [40, 9, 5, 130]), ([17, 1, 33], [17, 260, 70]),
                                      ([4, 6, 3], [2, 0, 300]), ([130, 1], [131, 1])])
def test_new_tokens(gpu, shape, new, lens):
    """Chunks of new tokens; also more of them than cached ones, whose first attend to nothing."""
    L = Layer(len(lens) + 10, *SHAPES[shape], page=16, rows=16 * (sum(-(-n // 16) for n in lens) + 2))
    table = L.table(lens)
    q = L.normal((sum(new) + 3, L.h, L.dh + L.dr))
    out = L.run(q, offsets(new), lens, table)
    check_attend(out[: sum(new)], *L.oracle(q, new, lens, L.slots_of(table)))
    assert bool((out[sum(new):] == 7).all())  # rows of no sequence


WIDE = 1 << 20  # tokens of capacity: enough for blocks of 128 rows wherever there are 48 rows a sequence


@pytest.mark.parametrize("shape", [s for s in SHAPES if s not in ("one", "d496", "tall")])
@pytest.mark.parametrize("new,lens", [([130, 1], [131, 1]), ([17, 70, 33], [17, 260, 70]), ([64, 0, 90], [500, 9, 60]),
                                      ([26], [63]), ([128, 128], [128, 129])])
def test_blocks_of_128_rows(gpu, shape, new, lens):
    """The same calls with a table wide enough that many rows are taken together."""
    L = Layer(len(lens) + 20, *SHAPES[shape], page=16, rows=16 * (sum(-(-n // 16) for n in lens) + 2))
    table = L.table(lens, WIDE // 16)
    q = L.normal((sum(new) + 3, L.h, L.dh + L.dr))
    out = L.run(q, offsets(new), lens, table)
    check_attend(out[: sum(new)], *L.oracle(q, new, lens, L.slots_of(table)))
    assert bool((out[sum(new):] == 7).all())


@pytest.mark.parametrize("shape", ["kv64", "h16", "mla320", "h128"])
@pytest.mark.parametrize("new,lens", [([1], [40000]), ([1] * 3, [9000, 17, 12345]), ([9, 2], [9000, 5000])])
def test_long_contexts(gpu, shape, new, lens):
    L = Layer(30, *SHAPES[shape], page=64, rows=64 * (sum(-(-n // 64) for n in lens) + 2))
    table = L.table(lens)
    q = L.normal((sum(new), L.h, L.dh + L.dr))
    check_attend(L.run(q, offsets(new), lens, table), *L.oracle(q, new, lens, L.slots_of(table)))


@pytest.mark.parametrize("shape", ["odd", "h16", "h128"])
def test_many_sequences(gpu, shape):
    lens = [(37 * i) % 200 for i in range(300)]
    new = [min(n, i % 4) for i, n in enumerate(lens)]
    L = Layer(31, *SHAPES[shape], page=16, rows=16 * (sum(-(-n // 16) for n in lens) + 2))
    table = L.table(lens)
    q = L.normal((sum(new), L.h, L.dh + L.dr))
    check_attend(L.run(q, offsets(new), lens, table), *L.oracle(q, new, lens, L.slots_of(table)))


def test_largest_batch(gpu):
    L = Layer(32, 2, 16, 16, 32, 8, page=4, rows=4 * 4100)
    lens = [1 + i % 3 for i in range(4096)]
    table = L.table(lens)
    q = L.normal((4096, 2, 24))
    check_attend(L.run(q, None, lens, table), *L.oracle(q, [1] * 4096, lens, L.slots_of(table)))


@pytest.mark.parametrize("shape", ["h16", "h128"])
def test_contiguous_rows_and_clamped_lengths(gpu, shape):
    L = Layer(33, *SHAPES[shape], page=16, rows=16 * 12)
    q = L.normal((4, L.h, L.dh + L.dr))
    at = lambda b, n: b * 48 + np.arange(n)
    out = torch.empty((4, L.h, L.dv), dtype=BF, device="cuda")
    ws = B.alloc_workspace(B.quant_attend_workspace_size(L.dims, 4, 4, 3))
    for lens, held in (([48, 1, 0, 30], [48, 1, 0, 30]), ([1000, -5, 49, 2 ** 31 - 1], [48, 0, 48, 48])):
        B.quant_attend(L.dims, q, None, L.codes, L.scales, L.w_uk, L.w_uv, ints(lens), None, 3, ws, out)
        check_attend(out, *L.oracle(q, [1] * 4, held, at))
    B.quant_attend(L.dims, q, None, L.codes, L.scales, L.w_uk, L.w_uv, ints([5, 5, 5, 5]),
                   torch.empty((4, 0), dtype=I32, device="cuda"), 0, ws, out)
    assert bool((out == 0).all())  # a capacity of nothing


@pytest.mark.parametrize("new", [1, 30])
@pytest.mark.parametrize("shape", ["odd", "h16", "mla320", "h128"])
def test_bad_pages_stay_in_the_cache(gpu, shape, new):
    L = Layer(34, *SHAPES[shape], page=16, rows=16 * 6)
    table = torch.full((2, WIDE // 16), 3, dtype=I32, device="cuda")
    table[:, :2] = ints([-7, 6, 2 ** 31 - 1, -2 ** 31]).reshape(2, 2)
    q = L.normal((2 * new, L.h, L.dh + L.dr))
    held = np.array([[0, 5], [5, 0]])
    at = lambda b, n: held[b, np.arange(n) // 16] * 16 + np.arange(n) % 16
    check_attend(L.run(q, offsets([new, new]), [30, 32], table), *L.oracle(q, [new, new], [30, 32], at))


@pytest.mark.parametrize("wide", [0, WIDE])
@pytest.mark.parametrize("shape", ["odd", "h16", "h128"])
def test_offsets_out_of_order_stay_in_bounds(gpu, shape, wide):
    L = Layer(35, *SHAPES[shape], page=16, rows=16 * 6)
    table = L.table([30, 30, 20], wide // 16 if wide else None)
    q = L.normal((40, L.h, L.dh + L.dr))
    for cu in ([0, 30, 10, 40], [5, 2 ** 31 - 1, -3, 20], [40, 0, 40, 0], [-2 ** 31, -1, 0, 2 ** 31 - 1], [0, 0, 0, 0]):
        L.run(q, ints(cu), [30, 30, 20], table)
    torch.cuda.synchronize()


@pytest.mark.parametrize("wide", [0, WIDE])
@pytest.mark.parametrize("shape", ["odd", "h16", "mla320", "h128"])
def test_rows_that_stand_for_nan_reach_only_those_that_attend_to_them(gpu, shape, wide):
    L = Layer(36, *SHAPES[shape], page=16, rows=16 * 20)
    lens, new = [40, 100, 33], [6, 20, 1]
    table = L.table(lens, wide // 16 if wide else None)
    at = L.slots_of(table)
    for b, j in ((0, 37), (1, 85), (2, 32)):
        slot = int(at(b, lens[b])[j])
        L.scales[slot] = 255
        L.codes[slot, : L.dc] = 0
    # whatever stands behind a sequence's last token, and in pages that it does not name, is not looked at
    used = np.concatenate([at(b, n) for b, n in enumerate(lens)])
    rest = torch.ones(L.rows, dtype=torch.bool, device="cuda")
    rest[torch.from_numpy(used).cuda()] = False
    L.codes[rest], L.scales[rest] = 0x7F, 255
    q = L.normal((sum(new), L.h, L.dh + L.dr))
    out = L.run(q, offsets(new), lens, table)
    want, size = L.oracle(q, new, lens, at)
    nan = np.isnan(want).all((1, 2))
    assert nan.tolist() == [i >= 3 for i in range(6)] + [i >= 5 for i in range(20)] + [True]
    check_attend(out, want, size)


@pytest.mark.parametrize("wide", [0, WIDE])
@pytest.mark.parametrize("shape", ["odd", "h16", "mla320", "h128"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_not_finite_keys(gpu, shape, value, wide):
    """A RoPE key that is not finite reaches only the rows that attend to it."""
    L = Layer(37, *SHAPES[shape], page=16, rows=16 * 20)
    lens, new = [50, 30], [10, 4]
    table = L.table(lens, wide // 16 if wide else None)
    slot = int(L.slots_of(table)(0, 50)[44])  # seen by the new tokens 4 .. 9 of the first
    L.codes[slot, L.dc: L.dc + 2] = torch.tensor([value], dtype=BF).view(U8).cuda()
    q = L.normal((14, L.h, L.dh + L.dr))
    out = L.run(q, offsets(new), lens, table)
    rows = cache_rows(L.codes, L.scales, L.dc)
    with np.errstate(invalid="ignore", over="ignore"):
        want, size = L.oracle(q, new, lens, L.slots_of(table), rows)
    seen = list(range(4, 10))
    rest = [i for i in range(14) if i not in seen]
    check_attend(out[rest], want[rest], size[rest])
    got = out[seen].double().cpu().numpy()
    # a score of -inf weighs nothing, one of +inf or NaN makes the head's row NaN
    assert np.array_equal(np.isnan(got), np.isnan(want[seen]))


@pytest.mark.parametrize("wide", [0, WIDE])
@pytest.mark.parametrize("shape", ["kv64", "h16", "mla320", "h128"])
def test_scales_of_any_size(gpu, shape, wide):
    """Rows of magnitudes from 2^-20 to 2^9 side by side; scores far apart."""
    L = Layer(38, *SHAPES[shape], page=16, rows=16 * 30)
    L.scales.copy_((127 + torch.randint(-20, 2, (L.rows,), generator=L.g, device="cuda")).to(U8))
    lens, new = [300, 50], [3, 11]
    table = L.table(lens, wide // 16 if wide else None)
    q = L.normal((14, L.h, L.dh + L.dr), 0.02)
    check_attend(L.run(q, offsets(new), lens, table), *L.oracle(q, new, lens, L.slots_of(table)))


@pytest.mark.parametrize("shape", ["h16", "h128"])
def test_a_workspace_of_a_larger_call_and_another_stream(gpu, shape):
    L = Layer(39, *SHAPES[shape], page=16, rows=16 * 40)
    ws = B.alloc_workspace(B.quant_attend_workspace_size(L.dims, 64, 200, 50)).fill_(0xFF)
    side = torch.cuda.Stream()
    for lens, new in (([100, 200], [20, 1]), ([33], [1]), ([5, 100, 200, 60], [5, 0, 7, 60])):
        table = L.table(lens)
        q = L.normal((sum(new), L.h, L.dh + L.dr))
        first = L.run(q, offsets(new), lens, table, ws=ws)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            second = L.run(q, offsets(new), lens, table, ws=ws)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(first, second)
        check_attend(first, *L.oracle(q, new, lens, L.slots_of(table)))


@pytest.mark.parametrize("shape", ["odd", "h16", "mla320"])
def test_decode_is_the_bf16_decode_of_the_same_values(gpu, shape):
    """eg_mla_decode over the rows read back, with a gate of ones, within both calls' roundings."""
    L = Layer(40, *SHAPES[shape], page=16, rows=16 * 40)
    lens = [1, 100, 333]
    table = L.table(lens)
    q = L.normal((3, L.h, L.dh + L.dr))
    out = L.run(q, None, lens, table)
    width = table.shape[1]
    rows = torch.zeros((L.rows, L.dc + L.dr), dtype=BF, device="cuda")
    B.quant_read(L.dims, L.codes, L.scales, None, ints([0, L.rows]), torch.arange(L.rows // 16, device="cuda", dtype=I32)[None], rows)
    d = B.make_dims(num_heads=L.h, head_dim=L.dh, v_head_dim=L.dv, latent_dim=L.dc, rope_dim=L.dr, vocab_size=1, page_size=16)
    other = torch.empty_like(out)
    B.decode(d, q, rows, torch.zeros(L.rows, dtype=I32, device="cuda"), torch.ones((1, L.dc), dtype=BF, device="cuda"), L.w_uk,
             L.w_uv, ints(lens), table, width, B.alloc_workspace(B.decode_workspace_size(d, 3, width)), other)
    want, size = L.oracle(q, [1] * 3, lens, L.slots_of(table))
    check_attend(out, want, size)
    check_attend(other, want, size)
