"""eg_mla_qk_norm_rope against the formulas in 64 bits.

Bound of an element: half a step of the storage type, and fp32 errors relative to the largest value A of its row:
the mean of n squares is off by at most n 2^-24 (halved by the root), the few products and the rotation's two terms by a
step each, and sine and cosine by 2^-21 (the angle's rounding, pi 2^-24, and two steps of the functions)."""
import numpy as np
import pytest
import torch

import server_oracle as S
from paper_2509_16686_amd import binding as B
from parity import say

pytestmark = pytest.mark.gpu
I32 = torch.int32
LAYERS = {
    "h16": dict(h=16, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),
    "kv64": dict(h=12, dh=64, dv=64, dc=64, dr=64, dtype="bf16"),
    "mla320": dict(h=16, dh=128, dv=128, dc=320, dr=64, dtype="bf16"),
    "h128": dict(h=128, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),
    "odd": dict(h=5, dh=24, dv=8, dc=40, dr=8, dtype="bf16"),
    "wide": dict(h=3, dh=1024, dv=64, dc=8, dr=632, dtype="bf16"),
    "long": dict(h=2, dh=512, dv=64, dc=64, dr=128, dtype="bf16"),
    "tiny": dict(h=4, dh=32, dv=32, dc=32, dr=0, dtype="fp32"),
    "f32": dict(h=8, dh=64, dv=64, dc=128, dr=32, dtype="fp32"),
    "f32wide": dict(h=3, dh=1024, dv=64, dc=4, dr=636, dtype="fp32"),
    "f32small": dict(h=7, dh=4, dv=4, dc=4, dr=4, dtype="fp32"),
}


def check(got, ref, top, n, storage, what):
    """|got - ref| within the bound above; `top` the row's largest value, broadcast."""
    half = 2.0 ** -8 if storage == "bf16" else 2.0 ** -24
    fp32 = ((n / 2 + 8) * 2.0 ** -24 + 2.0 ** -21) * top
    bound = half * (np.abs(ref) + fp32) + fp32
    worst = float(np.max(np.abs(got - ref) / np.maximum(bound, 1e-300))) if ref.size else 0.0
    say(f"  {what}: worst err/bound={worst:.3f}")
    assert worst <= 1.0, what


def row_top(x, axis=-1):
    return np.abs(x).max(axis, keepdims=True) if x.shape[axis] else x


class Rows:
    def __init__(self, layer, n, fused=False, weights=True, seed=1, top=131072):
        self.L = L = S.Layer(**LAYERS[layer], page=16, pages=1, seed=seed)
        self.n, self.dq, self.row = n, L.dh + L.dr, L.dc + L.dr
        if fused:
            x = L.normal((n, L.h * self.dq + self.row + 16), 1.3)
            self.q, self.kv = x[:, : L.h * self.dq], x[:, L.h * self.dq + 16:]
        else:
            self.q, self.kv = L.normal((n, L.h, self.dq), 1.3), L.normal((n, self.row), 1.3)
        self.qw = L.normal((self.dq,), 0.2, 1.0) if weights else None
        self.cw = L.normal((L.dc,), 0.2, 1.0) if weights else None
        self.kw = L.normal((L.dr,), 0.2, 1.0) if weights and L.dr else None
        self.positions, self.ids = L.ints(top, n), L.ints(211, n)
        self.num = n + 5
        self.slots = torch.randperm(self.num, generator=L.g)[:n].to(I32).cuda()
        self.cache = torch.full((self.num, self.row), -3.0, dtype=L.dtype, device="cuda")
        self.id_cache = torch.full((self.num,), -3, dtype=I32, device="cuda")
        self.q_out = torch.full((n, L.h, self.dq), -3.0, dtype=L.dtype, device="cuda")

    def run(self, q=True, kv=True, **kw):
        B.qk_norm_rope(self.L.dims, self.q if q else None, self.q_out if q else None, self.kv if kv else None,
                       self.cache if kv else None, self.id_cache if kv else None, self.ids if kv else None, self.positions,
                       self.slots if kv else None, q_norm_w=self.qw, kv_norm_w=self.cw if kv else None,
                       k_norm_w=self.kw if kv else None, **kw)
        torch.cuda.synchronize()

    def refs(self, theta=10000.0):
        L, f = self.L, self.L.f64
        w = lambda t: None if t is None else f(t)  # noqa: E731
        q = S.norm(f(self.q).reshape(self.n, L.h, self.dq), w(self.qw))
        kv, pos = f(self.kv), self.positions.cpu().numpy()
        c, r = S.norm(kv[:, : L.dc], w(self.cw)), S.norm(kv[:, L.dc:], w(self.kw)) if L.dr else kv[:, L.dc:]
        rot = np.concatenate([q[..., : L.dh], S.rope(q[..., L.dh:], pos, theta)], -1)
        return (rot, row_top(q)), (np.concatenate([c, S.rope(r, pos, theta)], 1),
                                   np.concatenate([np.broadcast_to(row_top(c), c.shape), np.broadcast_to(row_top(r), r.shape)], 1))

    def check(self, q=True, kv=True, theta=10000.0):
        (qr, qt), (kr, kt) = self.refs(theta)
        L, slots = self.L, self.slots.cpu().numpy()
        if q:
            check(L.f64(self.q_out).reshape(qr.shape), qr, qt, self.dq, L.storage, "q")
        else:
            assert bool((self.q_out == -3).all())
        cache, ids = L.f64(self.cache), self.id_cache.cpu().numpy()
        written = np.zeros(self.num, dtype=bool)
        if kv:
            ok = (slots >= 0) & (slots < self.num)
            check(cache[slots[ok]], kr[ok], kt[ok], L.dc, L.storage, "kv")
            assert np.array_equal(ids[slots[ok]], self.ids.cpu().numpy()[ok])
            written[slots[ok]] = True
        assert (cache[~written] == -3).all() and (ids[~written] == -3).all()  # other rows as they were


@pytest.mark.parametrize("layer", sorted(LAYERS))
@pytest.mark.parametrize("n", [1, 3, 64])
def test_matches_the_formulas(gpu, layer, n):
    say(f"qk_norm_rope {layer} n={n}")
    r = Rows(layer, n)
    r.run()
    r.check()


@pytest.mark.parametrize("layer", ["h16", "kv64", "f32", "odd"])
@pytest.mark.parametrize("weights", [True, False])
def test_strided_rows_of_one_projection(gpu, layer, weights):
    say(f"qk_norm_rope fused {layer} weights={weights}")
    r = Rows(layer, 37, fused=True, weights=weights)
    r.run()
    r.check()


@pytest.mark.parametrize("layer,n", [("h16", 700), ("h128", 300), ("tiny", 5000), ("kv64", 1030)])
def test_many_tokens(gpu, layer, n):
    say(f"qk_norm_rope {layer} n={n}")
    r = Rows(layer, n)
    r.run()
    r.check()


@pytest.mark.parametrize("layer", ["h16", "f32"])
def test_far_and_negative_positions(gpu, layer):
    say(f"qk_norm_rope positions {layer}")
    r = Rows(layer, 8)
    r.positions = torch.tensor([0, 1, 2 ** 31 - 1, 2 ** 30 + 7, 1048576, -1, -(2 ** 31), 131071], dtype=I32, device="cuda")
    r.run()
    r.check()


@pytest.mark.parametrize("theta", [500000.0, 1.0, 0.5, 1e30])
def test_other_frequencies(gpu, theta):
    say(f"qk_norm_rope theta={theta}")
    r = Rows("f32", 9, top=5000)
    r.run(rope_theta=theta)
    r.check(theta=float(np.float32(theta)))


def test_queries_or_keys_alone(gpu):
    say("qk_norm_rope alone")
    r = Rows("h16", 11)
    r.run(kv=False)
    r.check(kv=False)
    r = Rows("h16", 11)
    r.run(q=False)
    r.check(q=False)


@pytest.mark.parametrize("layer", ["h16", "h128", "wide", "f32"])
@pytest.mark.parametrize("weights", [True, False])
def test_in_place(gpu, layer, weights):
    say(f"qk_norm_rope in place {layer}")
    r = Rows(layer, 33, weights=weights)
    r.run()
    apart = r.q_out.clone()
    r.q_out = r.q
    r.run(kv=False)
    assert torch.equal(r.q.reshape(apart.shape), apart)


def test_slots_outside_the_cache_are_skipped(gpu):
    say("qk_norm_rope slots")
    r = Rows("h16", 6)
    r.slots = torch.tensor([-1, 3, r.num, 2 ** 31 - 1, 0, -(2 ** 31)], dtype=I32, device="cuda")
    r.run()
    r.check()


def test_infinite_and_nan_rows_stay_in_their_rows(gpu):
    say("qk_norm_rope non-finite")
    r = Rows("h16", 4)
    r.q[1, 2, 5], r.q[2, 0, 130], r.kv[3, 7] = float("inf"), float("nan"), float("nan")
    r.run()
    bad = ~torch.isfinite(r.q_out).all(-1)
    assert bad.nonzero().tolist() == [[1, 2], [2, 0]]
    assert (~torch.isfinite(r.cache[r.slots.long()]).all(-1)).nonzero().flatten().tolist() == [3]


def test_no_tokens(gpu):
    r = Rows("h16", 0)
    r.run()
    r.check()


def test_key_rows_are_the_append_ones(gpu):
    # the same projected rows through eg_mla_append: an identity projection of exact bf16 values
    say("qk_norm_rope against append")
    r = Rows("h16", 40)
    cache, ids = r.cache.clone(), r.id_cache.clone()
    eye = torch.eye(r.row, dtype=torch.bfloat16, device="cuda")
    r.kw = None
    B.append(r.L.dims, r.kv, r.ids, r.positions, r.slots, eye, r.cw, cache, ids)
    r.run()
    assert torch.equal(ids, r.id_cache)
    # sums in another order: a rounding apart at most
    a, b = r.L.f64(cache), r.L.f64(r.cache)
    assert np.all(np.abs(a - b) <= 2.0 ** -7 * np.abs(b) + 1e-6)
