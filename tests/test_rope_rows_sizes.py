"""Row rotations of more heads than their kernel's 32-bit numbers reach are refused on the host."""
import ctypes

import pytest

from paper_2509_16686_amd import binding as B


@pytest.mark.parametrize("heads", [(1 << 30) + 1, 2 ** 31 - 2048, 2 ** 31 - 1])
@pytest.mark.parametrize("dim,rd", [(1, 0), (2, 2)])
def test_heads_past_the_numbering(heads, dim, rd):
    rope = B.make_rope()
    at = lambda i: ctypes.c_void_p((i + 1) << 40)
    got = B.lib().eg_mla_rope_rows(ctypes.byref(rope), B.BF16, 1, heads, dim, 0, rd, at(0), 0, dim, at(1), 0, at(2), 0, dim, None)
    assert got == B.ERR_UNSUPPORTED
