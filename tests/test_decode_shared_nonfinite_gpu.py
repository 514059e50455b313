"""eg_mla_decode_shared with NaN and infinities among its inputs: what the softmax over them makes of it is not finite,
and nothing else changes (zeros are for sequences without tokens)."""
import numpy as np
import pytest
import torch

from paper_2509_16686_amd import binding as B
from parity import assert_close, say
from test_decode_shared_gpu import LAYERS, Case

pytestmark = pytest.mark.gpu
LAYERS.update({
    "h64dc512": dict(h=64, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),
    "h128dc128": dict(h=128, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),
})
KINDS = ["h16", "mla320", "h128", "h64dc512", "h32dc512", "h128dc128", "dv64", "kv64", "h5", "rope128", "f32", "f32wide"]
# one partial row or a few, with and without own tokens
SHAPES = [(20, [5, 0, 70]), (20, [0, 0, 0]), (777, [5, 0, 130]), (0, [40, 3, 130])]


def check(got, ref, lost, storage, what):
    """`lost` [B, H]: rows that are not finite; the others as in `ref`."""
    bad = ~np.isfinite(got)
    assert np.array_equal(bad.any(2), lost), f"{what}: rows {np.argwhere(bad.any(2) != lost).tolist()}"
    keep = ~lost
    if keep.any():
        assert_close(got[keep], ref[keep], storage, what)


@pytest.mark.parametrize("layer", KINDS)
@pytest.mark.parametrize("prefix,lens", SHAPES)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_query(gpu, layer, prefix, lens, value):
    say(f"decode_shared query {value} {layer} prefix={prefix} lens={lens}")
    c = Case(layer, prefix, lens, extra_pages=2)
    ref, h = c.ref(), c.L.h
    lost = np.zeros((3, h), dtype=bool)
    for b, head in [(0, 0), (0, h - 1), (1, h // 2), (2, h // 3)]:
        c.q[b, head, 3] = value
        lost[b, head] = prefix + lens[b] > 0
    check(c.run(), ref, lost, c.L.storage, layer)


@pytest.mark.parametrize("layer", KINDS)
@pytest.mark.parametrize("prefix,lens", SHAPES[:3])
def test_prefix_row(gpu, layer, prefix, lens):
    say(f"decode_shared prefix row NaN {layer} prefix={prefix} lens={lens}")
    c = Case(layer, prefix, lens, extra_pages=2)
    last = prefix - 1
    c.L.cache[int(c.prefix_table[last // c.page]) * c.page + last % c.page, 1] = float("nan")
    got = c.run()
    assert np.isnan(got).any(2).all()  # every row attends to it


@pytest.mark.parametrize("layer", KINDS)
@pytest.mark.parametrize("prefix,lens", [SHAPES[0], SHAPES[2], SHAPES[3]])
def test_own_row(gpu, layer, prefix, lens):
    say(f"decode_shared own row NaN {layer} prefix={prefix} lens={lens}")
    c = Case(layer, prefix, lens, extra_pages=2)
    ref, at = c.ref(), lens[2] - 1
    c.L.cache[int(c.table[2, at // c.page]) * c.page + at % c.page, 1] = float("nan")
    lost = np.zeros((3, c.L.h), dtype=bool)
    lost[2] = True
    check(c.run(), ref, lost, c.L.storage, layer)


@pytest.mark.parametrize("layer", KINDS)
def test_rows_behind_the_last_token_are_not_read_into_it(gpu, layer):
    say(f"decode_shared NaN behind the last tokens {layer}")
    c = Case(layer, 70, [5, 0, 130], extra_pages=2)
    ref = c.ref()
    for pages, n in [(c.prefix_table, 70), (c.table[0], 5), (c.table[2], 130)]:
        p = int(pages[n // c.page])
        c.L.cache[p * c.page + n % c.page:(p + 1) * c.page] = float("nan")
    check(c.run(), ref, np.zeros((3, c.L.h), dtype=bool), c.L.storage, layer)
