"""Sums of eg_mla_quant_attend are held in 32 bits: with scores of zero and values that are small whole numbers every sum
over keys is exact, and the output is the mean rounded once to bf16."""
import numpy as np
import pytest

from quant_peaked import Peaked, decode, encode
from test_quant_peaked_gpu import ROWS_16, ROWS_128, run, stage

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lengths", ["any", "short"])
@pytest.mark.parametrize("rows", [16, 128])
@pytest.mark.parametrize("dc", ROWS_128)
def test_means(gpu, dc, rows, lengths):
    """Rows of many partial rows, and (all lengths but one short) of one to three."""
    shape, b, new = (ROWS_16 if rows == 16 else ROWS_128)[dc]
    lens = [4096 - 61 * i % 4000 if lengths == "any" or i == 0 else 20 + 37 * i % 90 for i in range(b)]
    P = Peaked(dc, *shape, [new] * b, lens, "rope", 32)
    r = np.random.default_rng(dc)
    P.q = [np.zeros_like(q) for q in P.q]
    values = [r.integers(-6, 14, x.shape).astype(np.float64) for x in P.lat]
    P.codes, P.scales = map(list, zip(*(encode(x) for x in values)))
    assert all(np.array_equal(decode(c, s), x) for c, s, x in zip(P.codes, P.scales, values))
    sums = [np.cumsum(x, 0) for x in values]  # (whole numbers: exact)
    means = np.array([sums[k][n - new + i] / (n - new + i + 1) for k, n in enumerate(lens) for i in range(new)])
    want = means[:, P.pick_v]
    dims, args = stage(P, dc)
    got = run(P, dims, args).double().cpu().numpy()
    # the sum (below 2^16) and the count are exact in fp32, the quotient is off by 2^-22 of it, its two bf16 halves by 2^-17,
    # the output by half a step of its own power of two
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(want), 2.0 ** -60))) - 7)
    off = np.abs(got - want) / (step / 2 + 2.0 ** -16 * np.abs(want))
    at = np.unravel_index(off.argmax(), off.shape)
    assert off.max() <= 1, f"{off.max()} of the bound at {at}: {got[at]}, {want[at]}; {(off > 1).mean()} of the values"
