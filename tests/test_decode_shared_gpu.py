"""eg_mla_decode_shared against softmax attention over each sequence's prefix and own tokens in 64 bits, at the bars of
the decode (parity.py), and against eg_mla_decode on tables that name the prefix's pages for every sequence."""
import numpy as np
import pytest
import torch

import server_oracle as S
from paper_2509_16686_amd import binding as B
from parity import assert_close, say

pytestmark = pytest.mark.gpu
I32 = torch.int32
LAYERS = {
    "h16": dict(h=16, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),
    "mla320": dict(h=16, dh=128, dv=128, dc=320, dr=64, dtype="bf16"),
    "h128": dict(h=128, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),
    "h32dc512": dict(h=32, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),
    "h48": dict(h=48, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),
    "dv64": dict(h=16, dh=64, dv=64, dc=128, dr=64, dtype="bf16"),       # general merge
    "kv64": dict(h=12, dh=64, dv=64, dc=64, dr=64, dtype="bf16"),        # fp32 matrix-core kernel
    "h5": dict(h=5, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),        # heads that fill no 16
    "rope128": dict(h=6, dh=64, dv=40, dc=32, dr=128, dtype="bf16"),     # vector kernel
    "tiny": dict(h=4, dh=32, dv=32, dc=32, dr=0, dtype="fp32"),
    "f32": dict(h=8, dh=64, dv=64, dc=128, dr=32, dtype="fp32"),
    "f32wide": dict(h=3, dh=64, dv=72, dc=400, dr=0, dtype="fp32"),      # vector kernel
}


class Case:
    def __init__(self, layer, prefix, lens, page=64, extra_pages=0, seed=3, factor=1.0, own_width=None, scale=0.0):
        self.lens, self.prefix, self.page = list(lens), prefix, page
        pages = S.ceil_div(prefix, page) + sum(S.ceil_div(n, page) for n in lens) + extra_pages + 1
        self.L = S.Layer(**LAYERS[layer], page=page, pages=pages, seed=seed, scale=scale)
        self.table, self.prefix_table = self.L.table(lens, own_width, S.ceil_div(prefix, page) + extra_pages)
        self.q = self.L.query(len(lens), factor)
        self.seq_lens = torch.tensor(lens, dtype=I32, device="cuda")
        self.prefix_len = torch.tensor([prefix], dtype=I32, device="cuda")
        self.out = torch.full((len(lens), self.L.h, self.L.dv), float("nan"), dtype=self.L.dtype, device="cuda")

    def run(self, ws=None, stream=None, own=True, pre=True):
        L, width = self.L, self.table.shape[1] if own else 0
        if ws is None:
            n = B.decode_shared_workspace_size(L.dims, len(self.lens), width, self.prefix_table.numel() if pre else 0)
            assert n > 0
            ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # NaN bits: nothing there is read before it is written
        B.decode_shared(L.dims, self.q, L.cache, L.ids, L.gate, L.w_uk, L.w_uv, self.prefix_len if pre else None,
                        self.prefix_table if pre else None, self.seq_lens if own else None, self.table if own else None,
                        width, ws, self.out, stream=stream)
        torch.cuda.synchronize()
        return L.f64(self.out)

    def ref(self, prefix=None, lens=None):
        L = self.L
        n = self.prefix if prefix is None else prefix
        lens = self.lens if lens is None else lens
        shared, t = L.rows(self.prefix_table.cpu(), n), self.table.cpu()
        return L.attend(self.q, lambda b: np.concatenate([shared, L.rows(t[b].clamp(min=0), lens[b])]))

    def check(self, what, **kw):
        say(f"decode_shared {what}")
        got = self.run(**kw)
        assert_close(got, self.ref(), self.L.storage, what)


@pytest.mark.parametrize("layer", sorted(LAYERS))
@pytest.mark.parametrize("prefix,lens", [(1, [1]), (300, [5, 0, 130]), (777, [1, 64, 65, 0, 200, 3, 17])])
def test_matches_attention_over_both(gpu, layer, prefix, lens):
    Case(layer, prefix, lens).check(f"{layer} prefix={prefix} lens={lens}")


@pytest.mark.parametrize("layer", ["h16", "h128", "mla320"])
@pytest.mark.parametrize("batch", [1, 2, 3, 4, 5, 8, 9, 16, 17, 31, 33])
def test_batches(gpu, layer, batch):
    lens = [(37 * b) % 90 for b in range(batch)]
    Case(layer, 333, lens, page=16).check(f"{layer} batch={batch}")


@pytest.mark.parametrize("layer", ["h16", "h128", "kv64", "f32"])
@pytest.mark.parametrize("prefix", [31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 513])
def test_prefix_ends(gpu, layer, prefix):
    Case(layer, prefix, [9, 70], page=24).check(f"{layer} prefix={prefix}")


@pytest.mark.parametrize("layer,prefix,batch", [("h16", 20000, 3), ("h16", 5000, 40), ("h128", 4100, 6), ("mla320", 6000, 5),
                                                ("kv64", 9000, 3), ("f32", 5000, 3)])
def test_long_prefixes(gpu, layer, prefix, batch):
    Case(layer, prefix, [50 * b for b in range(batch)], factor=1.5).check(f"{layer} prefix={prefix} batch={batch}")


@pytest.mark.parametrize("layer", ["h16", "h128", "mla320", "tiny", "rope128"])
def test_empty_parts(gpu, layer):
    # no own tokens anywhere; no prefix token; neither: zeros
    Case(layer, 200, [0, 0, 0], own_width=3).check(f"{layer} no own tokens")
    c = Case(layer, 0, [40, 1, 0], extra_pages=2)
    c.check(f"{layer} no prefix token")
    assert not c.out[2].any()
    c = Case(layer, 0, [0, 0], extra_pages=2)
    assert not c.run().any()


@pytest.mark.parametrize("layer", ["h16", "h128", "tiny"])
def test_without_a_prefix_or_own_table(gpu, layer):
    c = Case(layer, 300, [40, 1, 0])
    say(f"decode_shared {layer} without own table")
    assert_close(c.run(own=False), c.ref(lens=[0, 0, 0]), c.L.storage, "own table missing")
    assert_close(c.run(pre=False), c.ref(prefix=0), c.L.storage, "prefix table missing")
    assert not c.run(own=False, pre=False).any()


@pytest.mark.parametrize("layer", ["h16", "h128", "f32"])
def test_lengths_are_clamped(gpu, layer):
    c = Case(layer, 128, [64, 30], own_width=2)
    say(f"decode_shared clamped {layer}")
    c.prefix_len.fill_(2 ** 31 - 1)  # two pages of 64
    c.seq_lens.copy_(torch.tensor([-4, 30], dtype=I32))
    assert_close(c.run(), c.ref(lens=[0, 30]), c.L.storage, "lengths beyond the tables")
    c.prefix_len.fill_(-1)
    assert_close(c.run(), c.ref(prefix=0, lens=[0, 30]), c.L.storage, "negative prefix")


@pytest.mark.parametrize("layer", ["h16", "h128", "f32"])
def test_bad_pages_and_ids_stay_in_the_cache(gpu, layer):
    c = Case(layer, 128, [64, 30])
    say(f"decode_shared bad pages {layer}")
    c.prefix_table[0], c.table[1, 0] = 2 ** 31 - 1, -5
    c.L.ids[::7], c.L.ids[1::7] = -1, 2 ** 31 - 1
    assert np.isfinite(c.run()).all()


@pytest.mark.parametrize("layer", ["h16", "h128"])
def test_peaked_softmax(gpu, layer):
    Case(layer, 1000, [100, 0, 300], factor=8.0, seed=5).check(f"{layer} query x8")


@pytest.mark.parametrize("layer", ["h16", "h128", "tiny"])
def test_equals_decode_over_whole_tables(gpu, layer):
    # a prefix of whole pages: the same tokens through eg_mla_decode
    c = Case(layer, 256, [33, 7, 64])
    say(f"decode_shared against decode {layer}")
    got = c.run()
    table = torch.cat([c.prefix_table[None, :].expand(3, -1), c.table], 1).contiguous()
    lens = c.seq_lens + 256
    out = torch.empty_like(c.out)
    ws = B.alloc_workspace(B.decode_workspace_size(c.L.dims, 3, table.shape[1]))
    B.decode(c.L.dims, c.q, c.L.cache, c.L.ids, c.L.gate, c.L.w_uk, c.L.w_uv, lens, table, table.shape[1], ws, out)
    torch.cuda.synchronize()
    assert_close(got, c.L.f64(out), c.L.storage, "shared against plain decode")


def test_contiguous_own_rows(gpu):
    # own tokens of sequence b at rows b * max_pages * P: the prefix on pages behind them
    say("decode_shared contiguous")
    L = S.Layer(**LAYERS["h16"], page=16, pages=20, seed=9)
    lens = [20, 48, 3]
    c = Case.__new__(Case)
    c.L, c.lens, c.prefix, c.page = L, lens, 100, 16
    c.table = torch.arange(9, dtype=I32, device="cuda").reshape(3, 3)
    c.prefix_table = torch.tensor([15, 9, 18, 12, 11, 10, 13], dtype=I32, device="cuda")
    c.q = L.query(3)
    c.seq_lens, c.prefix_len = torch.tensor(lens, dtype=I32, device="cuda"), torch.tensor([100], dtype=I32, device="cuda")
    c.out = torch.empty((3, 16, 128), dtype=torch.bfloat16, device="cuda")
    ref = c.ref()
    ws = B.alloc_workspace(B.decode_shared_workspace_size(L.dims, 3, 3, 7))
    B.decode_shared(L.dims, c.q, L.cache, L.ids, L.gate, L.w_uk, L.w_uv, c.prefix_len, c.prefix_table, c.seq_lens, None, 3,
                    ws, c.out)
    torch.cuda.synchronize()
    assert_close(L.f64(c.out), ref, "bf16", "contiguous own rows")


def test_another_softmax_scale(gpu):
    Case("h16", 200, [30, 2], scale=0.11).check("scale 0.11")


@pytest.mark.parametrize("layer", ["h16", "h128", "f32"])
def test_captured_and_replayed_with_other_lengths(gpu, layer):
    c = Case(layer, 700, [100, 30, 0, 64], own_width=4)
    say(f"decode_shared captured {layer}")
    ws = B.alloc_workspace(B.decode_shared_workspace_size(c.L.dims, 4, c.table.shape[1], c.prefix_table.numel()))
    torch.cuda.synchronize()
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=s):
        B.decode_shared(c.L.dims, c.q, c.L.cache, c.L.ids, c.L.gate, c.L.w_uk, c.L.w_uv, c.prefix_len, c.prefix_table,
                        c.seq_lens, c.table, c.table.shape[1], ws, c.out)
    for prefix, lens in [(700, [100, 30, 0, 64]), (3, [1, 1, 0, 1]), (0, [5, 0, 0, 0]), (650, [0, 0, 0, 0])]:
        c.prefix_len.fill_(prefix)
        c.seq_lens.copy_(torch.tensor(lens, dtype=I32))
        c.out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        replayed = c.L.f64(c.out)
        eager = c.run()
        assert np.array_equal(replayed, eager)
        assert_close(replayed, c.ref(prefix=prefix, lens=lens), c.L.storage, f"replay {prefix} {lens}")


def test_two_calls_at_once_with_their_own_workspaces(gpu):
    say("decode_shared two streams")
    cases = [Case("h16", 900, [100, 30, 0, 64], seed=11), Case("h128", 500, [40, 3], seed=12)]
    want = [c.run() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    wss = [B.alloc_workspace(B.decode_shared_workspace_size(c.L.dims, len(c.lens), c.table.shape[1], c.prefix_table.numel()))
           for c in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s, ws in zip(cases, streams, wss):
            B.decode_shared(c.L.dims, c.q, c.L.cache, c.L.ids, c.L.gate, c.L.w_uk, c.L.w_uv, c.prefix_len, c.prefix_table,
                            c.seq_lens, c.table, c.table.shape[1], ws, c.out, stream=s)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert np.array_equal(c.L.f64(c.out), w)
