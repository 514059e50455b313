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


def stage(P, seed):
    """(dims, arguments of quant_attend) of the case, its rows in random pages."""
    r = np.random.default_rng(seed)
    pages = [-(-n // PAGE) for n in P.lens]
    width, order = max(pages), r.permutation(sum(pages) + 3)
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
        rope = torch.from_numpy(P.rope[b]).to(BF).contiguous().view(torch.uint8).numpy()
        codes[slot, P.dc:] = rope.reshape(len(j), 2 * P.dr)
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


def check(P, seed):
    dims, args = stage(P, seed)
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
