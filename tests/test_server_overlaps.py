"""Outputs and workspaces that overlap inputs or one another are refused on the host (pointers that nothing reads)."""
import ctypes

import pytest

from paper_2509_16686_amd import binding as B

MB = 1 << 20
L = dict(num_heads=2, head_dim=64, v_head_dim=64, latent_dim=64, rope_dim=64, vocab_size=100, page_size=16)
ROW, SLOTS, NB, W, PRE = 128 * 2, 64, 3, 2, 4  # bytes of a cache row; cache rows; sequences; own and prefix pages


def at(i, off=0):
    return ctypes.c_void_p(MB * 16 * (i + 1) + off)


def call(name, args, change, dims):
    return getattr(B.lib(), name)(*{**args, **change, "dims": ctypes.byref(dims)}.values())


# each input's bytes; an output may begin where one ends
Q, W_UK, W_UV, GATE = NB * 2 * 128 * 2, 2 * 64 * 64 * 2, 2 * 64 * 64 * 2, 100 * 64 * 2
SHARED = dict(dims=None, batch=NB, q=at(0), cache=at(1), ids=at(2), gate=at(3), w_uk=at(4), w_uv=at(5), prefix_len=at(6),
              prefix_table=at(7), prefix_pages=PRE, lens=at(8), table=at(9), width=W, num_slots=SLOTS, ws=at(10),
              ws_bytes=8 * MB, out=at(11), stream=None)
SHARED_INPUTS = [(0, Q), (1, SLOTS * ROW), (2, SLOTS * 4), (3, GATE), (4, W_UK), (5, W_UV), (6, 4), (7, PRE * 4), (8, NB * 4),
                 (9, NB * W * 4)]
OUT = NB * 2 * 64 * 2


@pytest.mark.parametrize("i,size", SHARED_INPUTS)
def test_decode_shared(i, size):
    d = B.make_dims(**L)
    need = B.decode_shared_workspace_size(d, NB, W, PRE)
    first, last = 16 - OUT, (size - 1) // 16 * 16  # the out rows that end in the input's first bytes, or begin in its last
    for off in (first, 0, last):
        assert call("eg_mla_decode_shared", SHARED, dict(out=at(i, off)), d) == B.ERR_INVALID_ARG
    for off in (256 - need // 256 * 256, 0, (size - 1) // 256 * 256):
        assert call("eg_mla_decode_shared", SHARED, dict(ws=at(i, off)), d) == B.ERR_INVALID_ARG


def test_decode_shared_outputs():
    d = B.make_dims(**L)
    need = B.decode_shared_workspace_size(d, NB, W, PRE)
    for off in (16 - OUT, 0, (need - 1) // 16 * 16):
        assert call("eg_mla_decode_shared", SHARED, dict(out=at(10, off)), d) == B.ERR_INVALID_ARG


MEANS = dict(dims=None, batch=NB, cache=at(0), ids=at(1), gate=at(2), first=at(3), lens=at(4), table=at(5), width=W,
             num_slots=SLOTS, means=at(6), stream=None)


@pytest.mark.parametrize("i,size", [(0, SLOTS * ROW), (1, SLOTS * 4), (2, GATE), (3, NB * 4), (4, NB * 4), (5, NB * W * 4)])
def test_page_means(i, size):
    d = B.make_dims(**L)
    for off in (16 - SLOTS // 16 * ROW, 0, (size - 1) // 16 * 16):
        assert call("eg_mla_page_means", MEANS, dict(means=at(i, off)), d) == B.ERR_INVALID_ARG


SCORES = dict(dims=None, batch=NB, q=at(0), w_uk=at(1), means=at(2), lens=at(3), table=at(4), width=W, num_slots=SLOTS, ws=at(5),
              ws_bytes=8 * MB, scores=at(6), stream=None)


@pytest.mark.parametrize("i,size", [(0, Q), (1, W_UK), (2, SLOTS // 16 * ROW), (3, NB * 4), (4, NB * W * 4)])
def test_page_scores(i, size):
    d = B.make_dims(**L)
    need = B.page_scores_workspace_size(d, NB)
    for off in (4 - NB * W * 4, 0, size - 4):
        assert call("eg_mla_page_scores", SCORES, dict(scores=at(i, off)), d) == B.ERR_INVALID_ARG
    for off in (256 - need // 256 * 256, 0, (size - 1) // 256 * 256):
        assert call("eg_mla_page_scores", SCORES, dict(ws=at(i, off)), d) == B.ERR_INVALID_ARG


def test_page_scores_outputs():
    d = B.make_dims(**L)
    need = B.page_scores_workspace_size(d, NB)
    for off in (4 - NB * W * 4, 0, need - 4):
        assert call("eg_mla_page_scores", SCORES, dict(scores=at(5, off)), d) == B.ERR_INVALID_ARG
