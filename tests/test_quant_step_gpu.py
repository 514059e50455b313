"""Steps of a server on the 8-bit cache, every operator in turn: page tables, rotated queries, rows written, attention;
directly, and captured once and replayed for steps of other sizes; and rows far into a large cache."""
import math

import numpy as np
import pytest
import torch

from paper_2509_16686_amd import binding as B
from quant_oracle import BF, I32, U8, Layer, cache_rows, check_attend, frequencies, ints, offsets, rotate

pytestmark = pytest.mark.gpu


class Server:
    """A batch of sequences served by the library's calls; buffers of a fixed size, as a captured step needs them."""

    def __init__(self, seed, h, dh, dc, dr, batch, width, most, half):
        self.L = Layer(seed, h, dh, dh, dc, dr, page=16, rows=16 * 64)
        self.b, self.width, self.most, self.half = batch, width, most, half
        z = lambda n: torch.zeros(n, dtype=I32, device="cuda")
        self.lens, self.new, self.next = z(batch), z(batch), z(batch)
        self.table = torch.full((batch, width), -1, dtype=I32, device="cuda")
        self.free, self.count, self.left = self.L.perm(64), ints([64]), z(1)
        self.cu, self.positions, self.slots = z(batch + 1), z(most), z(most)
        self.x = torch.zeros((most, h * (dh + dr) + dc + dr), dtype=BF, device="cuda")  # a fused projection's rows
        self.ids = z(most)
        self.q = torch.zeros((most, h, dh + dr), dtype=BF, device="cuda")
        self.out = torch.zeros((most, h, dh), dtype=BF, device="cuda")
        self.ws = B.alloc_workspace(B.quant_attend_workspace_size(self.L.dims, batch, most, width))
        self.rope = B.make_rope(layout=int(half), frequencies=B.rope_frequencies(dr, 8.0, 64), magnitude=1.1)
        self.kv_w, self.k_w = self.L.normal((dc,), 0.1, 1.0), self.L.normal((dr,), 0.1, 1.0)

    def step(self):
        L, d = self.L, self.L.dims
        h, dq = L.h, L.dh + L.dr
        B.page_plan(16, self.lens, self.new, self.table, self.free, self.count, self.next, self.cu, self.positions, self.slots,
                    self.left)
        B.rope_rows(self.rope, self.x[:, : h * dq].unflatten(1, (h, dq)), self.positions, self.q, rope_dim=L.dr)
        B.quant_write(d, self.rope, self.x[:, h * dq:], self.positions, self.slots, L.codes, L.scales, gate_table=L.gate,
                      token_ids=self.ids, kv_norm_w=self.kv_w, k_norm_w=self.k_w)
        B.quant_attend(d, self.q, self.cu, L.codes, L.scales, L.w_uk, L.w_uv, self.next, self.table, self.width, self.ws, self.out)
        self.lens.copy_(self.next)
        self.count.copy_(self.left)

    def feed(self, new):
        n = sum(new)
        self.new.copy_(ints(new))
        self.x[:n] = self.L.normal((n, self.x.shape[1]))
        self.ids[:n] = self.L.ints(300, n)

    def check(self, new):
        """The queries' rotation and the attention over what the cache holds, and what the slots got."""
        L, n = self.L, sum(new)
        lens = self.lens.tolist()
        assert self.cu.tolist() == [0] + list(np.cumsum(new))
        if n == 0:
            return
        pos = np.concatenate([np.arange(k - m, k) for k, m in zip(lens, new)])
        f = frequencies(L.dr, factor=8.0, trained=64)
        q = self.x[:n, : L.h * (L.dh + L.dr)].reshape(n, L.h, -1).double().cpu().numpy().copy()
        q[..., L.dh:] = rotate(q[..., L.dh:], pos, f, self.half, float(np.float32(1.1)))
        got = self.q[:n].double().cpu().numpy()
        assert (np.abs(got - q) <= 2.0 ** -8 * np.abs(q) + 2.0 ** -19 * np.abs(q).max()).all()
        at = L.slots_of(self.table)
        rows = cache_rows(L.codes, L.scales, L.dc)
        slots = self.slots[:n].tolist()
        assert slots == [int(s) for b, (k, m) in enumerate(zip(lens, new)) for s in at(b, k)[k - m:]]
        c = self.x[:n, L.h * (L.dh + L.dr):].double().cpu().numpy()
        norm = lambda x, w: x / np.sqrt((x * x).mean(1, keepdims=True) + 1e-6) * w.double().cpu().numpy()
        lat = norm(c[:, : L.dc], self.kv_w) * L.gate[self.ids[:n].long()].double().cpu().numpy()
        key = rotate(norm(c[:, L.dc:], self.k_w), pos, f, self.half, float(np.float32(1.1)))
        # a code is within half a step of 2^-4, or of the least code, 2^-9 of 448's power of two at the row's largest
        top = np.abs(lat).max(1, keepdims=True)
        assert (np.abs(rows[slots, : L.dc] - lat) <= 2.0 ** -4 * np.abs(lat) * (1 + 2.0 ** -15) + top * 2.0 ** -10 / 224).all()
        assert (np.abs(rows[slots, L.dc:] - key) <= 2.0 ** -8 * np.abs(key) + 2.0 ** -19 * np.abs(key).max()).all()
        check_attend(self.out[:n], *L.oracle(self.q[:n], new, lens, at, rows))


LAYERS = [(5, 40, 48, 24), (16, 128, 128, 64), (16, 128, 320, 64), (128, 128, 512, 64)]


@pytest.mark.parametrize("layer", LAYERS)
@pytest.mark.parametrize("half", [False, True])
def test_steps(gpu, layer, half):
    s = Server(1, *layer, batch=3, width=8, most=70, half=half)
    for new in ([40, 3, 1], [1, 1, 1], [0, 17, 2], [4, 4, 4], [33, 1, 0]):
        s.feed(new)
        s.step()
        s.check(new)


@pytest.mark.parametrize("layer", LAYERS)
def test_captured_step(gpu, layer):
    """One graph for steps of any size up to its own; rows of no sequence stay as they are; eager calls in between."""
    s = Server(2, *layer, batch=3, width=8, most=70, half=True)
    keep = [t.clone() for t in (s.lens, s.table, s.count, s.L.codes, s.L.scales)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.feed([1, 1, 1])
        s.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    for t, k in zip((s.lens, s.table, s.count, s.L.codes, s.L.scales), keep):
        t.copy_(k)
    other = Layer(3, *layer[:2], layer[1], *layer[2:], page=16, rows=16 * 8)
    table = other.table([50])
    q = other.normal((1, other.h, other.dh + other.dr))
    first = other.run(q, None, [50], table)
    for new in ([40, 3, 1], [1, 1, 1], [0, 0, 0], [20, 30, 2], [1, 1, 1], [4, 0, 4]):
        s.feed(new)
        s.out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        s.check(new)
        assert bool((s.out[sum(new):] == 7).all())
        assert torch.equal(other.run(q, None, [50], table), first)
    # the captured arithmetic is the direct call's
    again = torch.full_like(s.out, 7.0)
    B.quant_attend(s.L.dims, s.q, s.cu, s.L.codes, s.L.scales, s.L.w_uk, s.L.w_uv, s.lens, s.table, s.width, s.ws, again)
    assert torch.equal(again, s.out)


def test_graphs_that_share_a_workspace(gpu):
    a, b = (Server(seed, 16, 128, 128, 64, batch=3, width=8, most=70, half=False) for seed in (4, 5))
    b.ws = a.ws
    graphs = []
    for s in (a, b):
        keep = [t.clone() for t in (s.lens, s.table, s.count)]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s.step()
        graphs.append(g)
        for t, k in zip((s.lens, s.table, s.count), keep):
            t.copy_(k)
    for new_a, new_b in (([9, 1, 30], [1, 1, 1]), ([1, 1, 1], [40, 20, 9]), ([2, 2, 2], [1, 0, 3])):
        for s, new, g in ((a, new_a, graphs[0]), (b, new_b, graphs[1])):
            s.feed(new)
            g.replay()
            s.check(new)


@pytest.mark.parametrize("layer,rows", [((16, 128, 128, 64), (1 << 33) // 256 + 4096), ((128, 128, 512, 64), (1 << 32) // 640 + 4096)])
def test_rows_past_32_bits_of_bytes(gpu, layer, rows):
    """A cache of more than 4 (8) GiB: the pages in use are its last ones."""
    h, dh, dc, dr = layer
    rows = rows // 16 * 16
    L = Layer(6, h, dh, dh, dc, dr, page=16, rows=256)
    small = L.codes, L.scales
    L.codes = torch.empty((rows, dc + 2 * dr), dtype=U8, device="cuda")
    L.scales = torch.empty(rows, dtype=U8, device="cuda")
    L.codes[-256:], L.scales[-256:] = small
    base, lens, new = rows // 16 - 16, [100, 60], [5, 1]
    order = torch.randperm(16, generator=L.g, device="cuda").to(I32)
    table = torch.full((2, 7), -1, dtype=I32, device="cuda")
    table[0, :7], table[1, :4] = order[:7] + base, order[7:11] + base
    near = torch.where(table < 0, table, table - base)
    held = cache_rows(*small, dc)
    q = L.normal((6, h, dh + dr))
    check_attend(L.run(q, offsets(new), lens, table), *L.oracle(q, new, lens, L.slots_of(near), held))
    out = torch.empty((160, dc + dr), dtype=BF, device="cuda")
    B.quant_read(L.dims, L.codes, L.scales, None, offsets(lens), table, out)
    at = L.slots_of(near)
    assert np.array_equal(out.double().cpu().numpy(), np.concatenate([held[at(0, 100)], held[at(1, 60)]]))
    slots = ints([rows - 1, rows - 200])
    kv = out[:2].contiguous()
    B.quant_write(L.dims, None, kv, None, slots, L.codes, L.scales)
    got = cache_rows(L.codes[slots.long()], L.scales[slots.long()], dc)
    assert np.array_equal(got, kv.double().cpu().numpy())  # values on the grid keep themselves


def test_another_device_than_the_current_one_is_refused(gpu):
    L = Layer(7, 4, 64, 64, 64, 32, rows=64)
    q = L.normal((1, 4, 96))
    with pytest.raises(ValueError):
        B.quant_attend(L.dims, q.cpu(), None, L.codes, L.scales, L.w_uk, L.w_uv, ints([5]), None, 1,
                       B.alloc_workspace(1 << 20), torch.empty((1, 4, 64), dtype=BF, device="cuda"))


def test_two_streams_with_their_own_workspaces(gpu):
    L = Layer(8, 16, 128, 128, 128, 64, page=16, rows=16 * 200)
    lens, new = [300, 500, 40], [4, 1, 40]
    table = L.table(lens)
    q = [L.normal((45, 16, 192)) for _ in range(2)]
    want = [L.run(x, offsets(new), lens, table) for x in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    cu, n = offsets(new), ints(lens)
    ws = [B.alloc_workspace(B.quant_attend_workspace_size(L.dims, 3, 45, table.shape[1])) for _ in range(2)]
    out = [torch.empty_like(want[0]) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            B.quant_attend(L.dims, q[i], cu, L.codes, L.scales, L.w_uk, L.w_uv, n, table, table.shape[1], ws[i], out[i], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
