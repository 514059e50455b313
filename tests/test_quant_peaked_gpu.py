"""eg_mla_quant_attend where single keys decide and running maxima grow within a run of tiles, in some rows and not in
others: against 64 bits within a bound that sees one key (quant_peaked.py), and bit for bit against itself."""
import numpy as np
import pytest
import torch

from paper_2509_16686_amd import binding as B
from quant_oracle import BF, I32, ints, offsets
from quant_peaked import Peaked

pytestmark = pytest.mark.gpu

PAGE = 64


def stage(P, seed, width=0):
    """(dims, arguments of quant_attend) of the case, its rows in random pages, in a table of at least `width` of them."""
    r = np.random.default_rng(seed)
    pages = [-(-n // PAGE) for n in P.lens]
    width, order = max(pages + [width]), r.permutation(sum(pages) + 3)
    table = np.full((len(P.lens), width), -1, dtype=np.int32)
    row = P.dc + 2 * P.dr
    codes = np.zeros((PAGE * len(order), row), dtype=np.uint8)
    scales = np.full(PAGE * len(order), 127, dtype=np.uint8)
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = order[at: at + n]
        at += n
        j = np.arange(P.lens[b])
        slot = table[b, j // PAGE].astype(np.int64) * PAGE + j % PAGE
        codes[slot, : P.dc], scales[slot] = P.codes[b], P.scales[b]
        if P.dr:
            codes[slot, P.dc:] = torch.from_numpy(P.rope[b]).to(BF).contiguous().view(torch.uint8).numpy()
    dims = B.make_dims(num_heads=P.h, head_dim=P.dh, v_head_dim=P.dv, latent_dim=P.dc, rope_dim=P.dr, vocab_size=1,
                       page_size=PAGE, dtype=B.BF16)
    dev = lambda x: torch.from_numpy(x).to(BF).cuda()
    return dims, (dev(np.concatenate(P.q)), offsets(P.new), torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(),
                  dev(P.w_uk), dev(P.w_uv), ints(P.lens), torch.from_numpy(table).to(I32).cuda(), width)


def run(P, dims, args):
    n, width = sum(P.new), args[-1]
    ws = B.alloc_workspace(B.quant_attend_workspace_size(dims, len(P.lens), n, width)).fill_(0xAB)
    out = torch.full((n, P.h, P.dv), 7.0, dtype=BF, device="cuda")
    B.quant_attend(dims, *args, ws, out)
    return out


def check(P, seed, width=0):
    dims, args = stage(P, seed, width)
    first = run(P, dims, args)
    for _ in range(3):
        assert torch.equal(run(P, dims, args), first)
    want, bound = P.attend()
    off = np.abs(first.double().cpu().numpy() - want) / bound
    assert off.max() <= 1, f"{off.max()} of the bound at {np.unravel_index(off.argmax(), off.shape)}"


# d_c: heads, d_h, d_v, d_c, d_r; sequences, new tokens of each: blocks of 128 query rows (48 rows a sequence and more),
# four tiles a run and more (tiles of 64 tokens and 512 runs up to d_c 128, of 32 and 256 runs above)
ROWS_128 = {64: ((12, 64, 64, 64, 64), 24, 11), 128: ((16, 128, 128, 128, 64), 24, 8), 144: ((16, 64, 136, 144, 64), 8, 8),
            320: ((16, 128, 128, 320, 64), 8, 8), 512: ((16, 128, 128, 512, 64), 8, 8)}
# blocks of 16 rows (fewer rows a sequence), three tiles a run and more (of 128 tokens up to d_c 128, of 64 above; 512 runs)
ROWS_16 = {64: ((12, 64, 64, 64, 64), 40, 2), 128: ((16, 128, 128, 128, 64), 40, 1), 144: ((16, 64, 136, 144, 64), 24, 2),
           320: ((16, 128, 128, 320, 64), 24, 1), 512: ((16, 128, 128, 512, 64), 24, 1)}


@pytest.mark.parametrize("dc", ROWS_128)
@pytest.mark.parametrize("peaks", ["rope", "latent"])
def test_blocks_of_128_rows(gpu, dc, peaks):
    shape, b, new = ROWS_128[dc]
    lens = [4096 - 37 * i % 200 for i in range(b)]
    check(Peaked(dc, *shape, [new] * b, lens, peaks, 32), dc)


@pytest.mark.parametrize("dc", ROWS_16)
@pytest.mark.parametrize("peaks", ["rope", "latent"])
def test_blocks_of_16_rows(gpu, dc, peaks):
    shape, b, new = ROWS_16[dc]
    lens = [4096 - 37 * i % 200 for i in range(b)]
    check(Peaked(dc, *shape, [new] * b, lens, peaks, 4), dc)


#                    h    d_h   d_v  d_c  d_r
ODD = {"dv7": (16, 128, 7, 128, 64), "dv33": (5, 64, 33, 48, 24), "h700": (700, 16, 1, 64, 8), "dv130": (16, 64, 130, 320, 64),
       "tall": (3, 1024, 1000, 512, 0), "h130": (130, 8, 12, 16, 0), "one": (1, 64, 64, 496, 8)}


@pytest.mark.parametrize("width", [0, 1 << 14])  # (a table of 2^20 tokens: blocks of 128 where there are 48 rows a sequence)
@pytest.mark.parametrize("shape", ODD)
def test_odd_shapes(gpu, shape, width):
    check(Peaked(70, *ODD[shape], [3, 60, 1, 17], [70, 333, 64, 17], "latent", 4), 70, width)
