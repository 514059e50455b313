"""eg_mla_decode_shared where its kernels change over: heads that fill no row block or several, own tokens on the wide
kernel, own splits at the list's end, many and few tiles, caches past 32-bit byte offsets."""
import numpy as np
import pytest
import torch

import server_oracle as S
from paper_2509_16686_amd import binding as B
from parity import assert_close, say
from test_decode_shared_gpu import LAYERS, Case

pytestmark = pytest.mark.gpu
I32 = torch.int32
LAYERS.update({
    "h64dc512": dict(h=64, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),     # own tokens on the wide kernel
    "h192dc512": dict(h=192, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),   # ... row blocks over two sequences
    "h256dc512": dict(h=256, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),   # two row blocks a sequence
    "h3dc512": dict(h=3, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),
    "h1": dict(h=1, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),
    "h128dc128": dict(h=128, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),
    "h20dc320": dict(h=20, dh=128, dv=128, dc=320, dr=64, dtype="bf16"),
})


@pytest.mark.parametrize("layer", ["h64dc512", "h192dc512", "h256dc512", "h3dc512", "h1", "h128dc128", "h20dc320"])
@pytest.mark.parametrize("prefix,lens", [(1, [1]), (500, [0, 33, 70, 1, 0]), (65, [600, 31, 32])])
def test_head_counts(gpu, layer, prefix, lens):
    Case(layer, prefix, lens, page=16).check(f"{layer} prefix={prefix} lens={lens}")


@pytest.mark.parametrize("layer", ["h64dc512", "h256dc512", "h128dc128"])
def test_parts_missing(gpu, layer):
    c = Case(layer, 300, [40, 1, 0])
    say(f"decode_shared parts {layer}")
    assert_close(c.run(own=False), c.ref(lens=[0, 0, 0]), "bf16", "own table missing")
    assert_close(c.run(pre=False), c.ref(prefix=0), "bf16", "prefix table missing")
    c.prefix_len.fill_(0)
    assert_close(c.run(), c.ref(prefix=0), "bf16", "no prefix token")
    c.seq_lens.zero_()
    assert not c.run().any()


@pytest.mark.parametrize("layer", ["h128", "h256dc512"])
@pytest.mark.parametrize("lens", [[511, 512, 513, 31], [2000, 1], [0, 5000, 0]])
def test_own_tokens_of_the_fused_kernel(gpu, layer, lens):
    # its list holds 512 tokens of a work-group at a time
    Case(layer, 40, lens, page=64).check(f"{layer} fused own {lens}")


def test_long_own_tokens_of_one_split(gpu):
    # one prefix token: every work-group of the fused kernel but the first has own tokens only, several lists each
    c = Case("h128", 1, [9000] + [1] * 70, page=64)
    c.check("h128 own 9000 of 71 sequences")


@pytest.mark.parametrize("batch", [63, 64, 65, 80])
def test_own_splits_at_the_list_end(gpu, batch):
    # capacity 4096: own splits of up to 1024 tokens share the prefix's launch, longer ones do not
    lens = [4096, 4095, 1025, 1024, 1023, 0, 1] + [64 * (b % 7) for b in range(batch - 7)]
    Case("h16", 70, lens, page=64).check(f"h16 batch={batch} own capacity 4096")


def test_query_times_eight_in_every_tiled_width(gpu):
    for layer in ("h16", "mla320", "h64dc512", "h128"):
        Case(layer, 700, [100, 0, 31], factor=8.0, seed=7).check(f"{layer} query x8")


def test_many_tiles(gpu):
    # 64 row blocks and 257 tiles: more than share a launch with the own tokens; the reference on the GPU in 64 bits
    lens = [(b * 37) % 200 for b in range(64)]
    c = Case("h128dc128", 16448, lens, page=64, seed=8)
    say("decode_shared h128dc128 16448 x 64")
    got, L = c.run(), c.L
    pages = c.prefix_table.long()
    at = (pages[:, None] * 64 + torch.arange(64, device="cuda")).reshape(-1)[:16448]
    x = L.cache[at].double()
    x[:, : L.dc] *= L.gate[L.ids[at].long()].double()
    qf = torch.cat([torch.matmul(c.q.double().transpose(0, 1)[..., : L.dh], L.w_uk.double()).transpose(0, 1),
                    c.q.double()[..., L.dh:]], 2) * L.tau
    for b in (0, 5, 31, 63):
        own = torch.from_numpy(L.rows(c.table[b].cpu().clamp(min=0), lens[b])).cuda()
        key = torch.cat([x, own])
        o = torch.softmax(qf[b] @ key.T, 1) @ key[:, : L.dc]
        ref = torch.matmul(L.w_uv.double(), o[:, :, None])[:, :, 0].cpu().numpy()
        assert_close(got[b], ref, "bf16", f"sequence {b}")


@pytest.mark.parametrize("layer", ["h128", "h16", "h64dc512"])
def test_rows_past_32_bit_offsets(gpu, layer):
    # the cache's last pages, more than 4 GiB from its start
    say(f"decode_shared far rows {layer}")
    c = Case(layer, 200, [70, 3, 64], page=64)
    L, row = c.L, c.L.dc + c.L.dr
    far = (1 << 32) // (2 * row * 64) + 5  # pages in front
    cache = torch.zeros(((far + L.pages) * 64, row), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros((far + L.pages) * 64, dtype=I32, device="cuda")
    cache[far * 64:], ids[far * 64:] = L.cache, L.ids
    ref = c.ref()
    L.cache, L.ids = cache, ids
    c.prefix_table += far
    c.table[c.table >= 0] += far
    assert_close(c.run(), ref, "bf16", "far rows")
    # the same rows' page means and keys
    means = torch.zeros((far + L.pages, row), dtype=torch.bfloat16, device="cuda")
    B.page_means(L.dims, cache, ids, L.gate, None, c.seq_lens, c.table, c.table.shape[1], means)
    torch.cuda.synchronize()
    want = L.rows([int(c.table[2, 0])], 64).mean(0)
    got = L.f64(means[int(c.table[2, 0])])
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * (1 + 2.0 ** -20) * np.abs(want) + 1e-38)
    slots = torch.tensor([cache.shape[0] - 1, cache.shape[0], 5], dtype=I32, device="cuda")
    kv, pos = L.normal((3, row)), torch.zeros(3, dtype=I32, device="cuda")
    B.qk_norm_rope(L.dims, None, None, kv, cache, ids, pos, pos, slots)
    torch.cuda.synchronize()
    assert torch.equal(cache[-1], kv[0]) and torch.equal(cache[5], kv[2])  # position 0 turns nothing


@pytest.mark.parametrize("layer", ["h16", "h128", "h64dc512", "mla320", "kv64", "f32"])
def test_prefix_whose_scores_overflow_weighs_nothing(gpu, layer):
    # q^R . k^R overflows to -inf over the prefix and is zero over the own tokens
    c = Case(layer, 300, [40, 0, 70], page=16)
    say(f"decode_shared overflow {layer}")
    L = c.L
    L.cache[:, L.dc:] = 0
    for p in c.prefix_table.tolist():
        L.cache[p * 16:(p + 1) * 16, L.dc:] = 3e38
    c.q[..., L.dh:] = -3e38
    q = c.q.clone()
    got = c.run()
    c.q[..., L.dh:] = 0  # the reference over the own tokens alone
    ref = c.ref(prefix=0)
    c.q = q
    assert_close(got[[0, 2]], ref[[0, 2]], L.storage, "own tokens alone")
    assert not got[1].any()
