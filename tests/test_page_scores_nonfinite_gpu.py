"""eg_mla_page_scores with NaN and infinities in queries and means: the maximum over the heads of fp32 scores, NaN where
one of them is, on the matrix cores as on the vector path; and absorbed queries at the end of the fp32 range.

Finite scores: 1e-3 of the sum of the products' sizes is far above their error (about (d_h + d_c + d_r) 2^-24 of it) and
far below what a lost part of the query or a lost head makes."""
import numpy as np
import pytest
import torch

from parity import say
from test_page_select_gpu import LAYERS, Cache

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
KINDS = ["h16", "kv64", "mla320", "h128", "h37", "top", "odd", "f32"]


def reference(c, q):
    """(max over heads of each page's score, sum of the products' sizes) in 64 bits."""
    L = c.L
    q64, w, m, t = L.f64(q), L.f64(L.w_uk), L.f64(c.means), c.table.cpu().numpy()
    score = np.full((len(c.lens), c.width), -INF)
    size = np.zeros_like(score)
    with np.errstate(all="ignore"):
        for b, n in enumerate(c.lens):
            for j in range(-(-n // c.page)):
                row = m[t[b, j]]
                ql = (q64[b, :, : L.dh, None] * w).sum(1)  # (not a library product: NaN and infinity as they are)
                qf = np.concatenate([ql, q64[b, :, L.dh:]], 1)
                score[b, j] = np.max((qf * row).sum(1)) * L.tau
                size[b, j] = np.max(np.abs(qf * row).sum(1)) * L.tau
    return score, size


def check(c, q, what):
    say(f"page scores {what}")
    got = c.scores(q).double().cpu().numpy()
    ref, size = reference(c, q)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what
    edge = np.isinf(ref)
    assert np.array_equal(got[edge], ref[edge]), what
    fin = np.isfinite(ref)
    assert np.all(np.abs(got[fin] - ref[fin]) <= 1e-3 * size[fin] + 1e-30), what
    return ref


@pytest.mark.parametrize("layer", KINDS)
def test_query(gpu, layer):
    c = Cache(layer, [100, 333, 40, 17], 16)
    c.L.w_uk.abs_().add_(0.01)  # every product of one sign: an infinite one makes an infinite score, not a NaN
    c.means.abs_().add_(0.01)
    for name, at in [("latent", 3), ("rope", c.L.dh + 1)]:
        if at >= c.L.dh + c.L.dr:
            continue
        q, h = c.L.query(4), c.L.h
        q[0, h - 1, at], q[1, 0, at], q[2, h // 2, at] = INF, -INF, NAN
        ref = check(c, q, f"{layer} {name}")
        assert (ref[0, :7] == INF).all() and np.isfinite(ref[1, :21]).all() and np.isnan(ref[2, :3]).all()
        q[1, :, at] = -INF  # every head
        assert (check(c, q, f"{layer} {name} all heads")[1, :21] == -INF).all()


@pytest.mark.parametrize("layer", KINDS)
def test_means(gpu, layer):
    c = Cache(layer, [100, 333, 40, 17], 16)
    q = c.L.query(4)
    last = c.L.dc + c.L.dr - 1
    for (b, j), col, value in [((0, 1), 0, INF), ((0, 3), c.L.dc - 1, -INF), ((1, 0), 5, NAN), ((1, 20), last, INF),
                               ((2, 2), last, NAN), ((3, 0), 7, -INF)]:
        c.means[int(c.table[b, j]), col] = value
    ref = check(c, q, f"{layer} means")
    assert np.isinf(ref[0, [1, 3]]).all() and np.isnan(ref[1, 0]) and np.isnan(ref[2, 2])
    # infinite against an infinite query of either sign
    q[0, 0, 2], q[3, 0, 2] = INF, -INF
    check(c, q, f"{layer} means and queries")


@pytest.mark.parametrize("layer", ["h16", "kv64", "mla320", "h128", "h37"])
@pytest.mark.parametrize("sign", [1, -1])
def test_absorbed_query_past_the_largest_bf16_value(gpu, layer, sign):
    # q_lat = +-2^128 (1 - 2^-10), finite in fp32, over bf16's largest value 2^128 (1 - 2^-8) by more than half a step
    c = Cache(layer, [100, 40], 16)
    q = torch.zeros_like(c.L.query(2))
    c.L.w_uk.zero_()
    q[:, :, 0], q[:, :, 1] = sign * 2.0 ** 127 * (2 - 2.0 ** -7), sign * 2.0 ** 118 * 1.5
    c.L.w_uk[:, 0, 2], c.L.w_uk[:, 1, 2] = 1, 1
    c.means[:, 2] = 2.0 ** -100
    ref = check(c, q, f"{layer} near the end of the range")
    assert np.isfinite(ref[0, :7]).all()
