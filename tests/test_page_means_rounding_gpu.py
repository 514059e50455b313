"""eg_mla_page_means rounds a mean once to bf16: means next to the middle of two bf16 values go to the nearer one."""
import numpy as np
import pytest
import torch

from paper_2509_16686_amd import binding as B
from parity import say
from test_page_select_gpu import Cache

pytestmark = pytest.mark.gpu


def nearest_bf16(x):
    """float64 values rounded to 8 significant bits, ties to even (no underflow)."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def formed(c):
    B.page_means(c.L.dims, c.L.cache, c.L.ids, c.L.gate, None, c.seq_lens, c.table, c.width, c.means)
    torch.cuda.synchronize()
    return c.L.f64(c.means)


@pytest.mark.parametrize("layer", ["h16", "h128", "odd"])
def test_means_next_to_a_tie(gpu, layer):
    say(f"page means next to ties {layer}")
    c = Cache(layer, [2, 4], 16)
    L, p0, p1 = c.L, int(c.table[0, 0]), int(c.table[1, 0])
    # two tokens: products of two bf16 values, (twice) an odd multiple of 2^-8, and a rest of 2^-31 of either sign
    L.ids[p0 * 16], L.ids[p0 * 16 + 1] = 3, 4
    for col, (a, b, rest) in enumerate([(7 / 8, 37 / 16, -1), (7 / 8, 37 / 16, 1), (-7 / 8, 37 / 16, 1), (9 / 8, 29 / 16, 1),
                                        (9 / 8, 29 / 16, -1), (-9 / 8, 29 / 16, -1), (9 / 8, 29 / 16, 0)]):
        L.cache[p0 * 16, col], L.gate[3, col] = a, b
        L.cache[p0 * 16 + 1, col], L.gate[4, col] = rest * 2.0 ** -30, 1.0
    # four tokens of the RoPE key, which has no gate
    for k, (base, rest) in enumerate([(3 / 64, -1), (3 / 64, 1), (5 / 64, 1), (5 / 64, -1)]):
        for t, v in enumerate([4.0, base, rest * 2.0 ** -29, 0.0]):
            L.cache[p1 * 16 + t, L.dc + k] = v
    got = formed(c)
    want = {p0: L.rows([p0], 2).mean(0), p1: L.rows([p1], 4).mean(0)}
    near = np.abs(np.abs(want[p0][:6]) - np.array([259, 259, 259, 261, 261, 261]) / 256)
    assert np.all((near > 0) & (near < 2.0 ** -30))
    for p, mean in want.items():
        assert np.array_equal(got[p], nearest_bf16(mean))


@pytest.mark.parametrize("layer", ["h16", "kv64", "mla320", "h128", "odd", "top"])
def test_every_mean_is_the_nearest(gpu, layer):
    say(f"page means nearest {layer}")
    c = Cache(layer, [100, 333, 7, 64, 1], 16, seed=11)
    got = formed(c)
    for p, mean in c.mean_refs():
        assert np.array_equal(got[p], nearest_bf16(mean)), p


def test_non_finite_and_zero_means(gpu):
    say("page means non-finite")
    c = Cache("h16", [3], 16)
    p = int(c.table[0, 0])
    c.L.gate.fill_(1)
    rows = c.L.cache[p * 16:p * 16 + 3]
    rows[:, 0], rows[:, 1], rows[:, 2], rows[:, 3] = 0, float("inf"), float("nan"), 3.3895e38
    rows[1, 1] = 5
    got = formed(c)[p]
    assert got[0] == 0 and got[1] == np.inf and np.isnan(got[2]) and got[3] == float(rows[0, 3])
