"""eg_mla_decode_shared of 128-head blocks with a prefix shorter than the own tokens, whose work-groups follow those."""
import pytest

from parity import assert_close, say
from test_decode_shared_gpu import LAYERS, Case

pytestmark = pytest.mark.gpu
LAYERS["h256dc512"] = dict(h=256, dh=128, dv=128, dc=512, dr=64, dtype="bf16")


@pytest.mark.parametrize("layer", ["h128", "h256dc512"])
@pytest.mark.parametrize("prefix,lens,page", [(64, [4096], 64), (16, [4000, 1, 0, 33, 700], 16), (40, [31, 32, 33, 64], 64),
                                              (1, [9000, 8], 64), (256, [5000, 300, 0], 64)])
def test_matches_attention(gpu, layer, prefix, lens, page):
    Case(layer, prefix, lens, page=page).check(f"{layer} prefix={prefix} lens={lens}")


@pytest.mark.parametrize("layer", ["h128", "h256dc512"])
def test_wide_tables_with_few_tokens(gpu, layer):
    # as many splits as the tables' capacity asks for, nearly all of them without tokens
    say(f"decode_shared wide tables {layer}")
    c = Case(layer, 30, [5, 0, 70], own_width=200, extra_pages=3)
    assert_close(c.run(), c.ref(), "bf16", "few tokens")
    c.prefix_len.zero_()
    assert_close(c.run(), c.ref(prefix=0), "bf16", "no prefix token")
    c.seq_lens.zero_()
    assert not c.run().any()


@pytest.mark.parametrize("batch", [15, 17, 18, 19, 20, 22, 24, 26, 28])
def test_partial_rows_of_each_merge(gpu, batch):
    # 17 to 9 rows a sequence, around the change from one merge to the other
    Case("h128", 700, [(53 * b) % 140 for b in range(batch)], page=16).check(f"h128 batch={batch}")
