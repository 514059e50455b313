"""Calls of the operators around the decode that are refused on the host, before anything is enqueued: by the C entries
(pointers that nothing reads) and by the binding (tensors that the entries would misread)."""
import ctypes

import pytest
import torch

from paper_2509_16686_amd import binding as B

OK, ARG, UNSUP, WS = B.OK, B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED, B.ERR_WORKSPACE
BIG = 1 << 20  # made-up addresses, a MiB apart


def at(i, off=0):
    return ctypes.c_void_p(BIG * (i + 1) + off)


def dims(**kw):
    base = dict(num_heads=16, head_dim=128, v_head_dim=128, latent_dim=128, rope_dim=64, vocab_size=500, page_size=64)
    base.update(kw)
    return B.make_dims(**base)


PLAN = dict(batch=4, page_size=16, width=8, max_tokens=50, cached=at(0), new=at(1), base=at(2), table=at(3), free=at(4),
            count=at(5), cap=64, lens=at(6), cu=at(7), positions=at(8), slots=at(9), count_out=at(10), stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(batch=0), OK), (dict(batch=-1), ARG), (dict(batch=4097), UNSUP), (dict(page_size=0), ARG), (dict(width=-1), ARG),
    (dict(max_tokens=-1), ARG), (dict(cap=-1), ARG), (dict(width=1 << 27), ARG), (dict(max_tokens=(1 << 30) + 1), ARG),
    (dict(cap=(1 << 30) + 1), ARG), (dict(cached=None), ARG), (dict(new=None), ARG), (dict(table=None), ARG),
    (dict(free=None), ARG), (dict(count=None), ARG), (dict(lens=None), ARG), (dict(cu=None), ARG), (dict(positions=None), ARG),
    (dict(slots=None), ARG), (dict(count_out=None), ARG),
    (dict(lens=at(0)), ARG), (dict(lens=at(0, 12)), ARG), (dict(cu=at(1)), ARG), (dict(positions=at(2)), ARG),
    (dict(slots=at(4)), ARG), (dict(count_out=at(5)), ARG), (dict(positions=at(9, 4)), ARG), (dict(lens=at(3, 124)), ARG),
    (dict(count_out=at(4, 252)), ARG), (dict(cu=at(6, 12)), ARG),
])
def test_page_plan(change, expect):
    assert B.lib().eg_mla_page_plan(*{**PLAN, **change}.values()) == expect


RELEASE = dict(batch=4, page_size=16, width=8, lens=at(0), ended=at(1), table=at(2), free=at(3), count=at(4), cap=64,
               lens_out=at(5), count_out=at(6), stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(batch=0), OK), (dict(batch=-1), ARG), (dict(batch=4097), UNSUP), (dict(page_size=0), ARG), (dict(width=-1), ARG),
    (dict(cap=-1), ARG), (dict(width=1 << 27), ARG), (dict(lens=None), ARG), (dict(ended=None), ARG), (dict(table=None), ARG),
    (dict(free=None), ARG), (dict(count=None), ARG), (dict(lens_out=None), ARG), (dict(count_out=None), ARG),
    (dict(lens_out=at(0)), ARG), (dict(count_out=at(4)), ARG), (dict(free=at(2)), ARG), (dict(lens_out=at(3, 252)), ARG),
])
def test_page_release(change, expect):
    assert B.lib().eg_mla_page_release(*{**RELEASE, **change}.values()) == expect


# 8 tokens; rows of 16 * 192 and 192 bf16 values, a cache of 32 rows
QROW = 16 * 192
QK = dict(dims=None, n=8, q=at(0), q_stride=QROW, q_w=at(1), q_out=at(2), kv=at(3), kv_stride=192, kv_w=at(4), k_w=at(5),
          ids=at(6), positions=at(7), slots=at(8), theta=10000.0, cache=at(9), id_cache=at(10), num_slots=32, stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(n=0), OK), (dict(n=-1), ARG), (dict(num_slots=-1), ARG), (dict(theta=float("inf")), ARG), (dict(q=None, kv=None), ARG),
    (dict(positions=None), ARG), (dict(q_out=None), ARG), (dict(q_stride=QROW - 8), ARG), (dict(q_stride=QROW + 4), ARG),
    (dict(q_stride=(1 << 32) + 8), ARG), (dict(kv_stride=184), ARG), (dict(kv_stride=194), ARG), (dict(kv_stride=1 << 40), ARG),
    (dict(q=at(0, 8)), ARG), (dict(q_out=at(2, 2)), ARG), (dict(q_w=at(1, 4)), ARG), (dict(kv=at(3, 8)), ARG),
    (dict(kv_w=at(4, 8)), ARG), (dict(k_w=at(5, 8)), ARG), (dict(cache=at(9, 8)), ARG), (dict(ids=None), ARG),
    (dict(slots=None), ARG), (dict(cache=None), ARG), (dict(id_cache=None), ARG),
    (dict(q_out=at(0), q_stride=QROW + 192), ARG),       # in place needs the same rows
    (dict(q_out=at(0, 16)), ARG), (dict(q_out=at(3, 16)), ARG), (dict(cache=at(3)), ARG), (dict(cache=at(0, 16)), ARG),
    (dict(cache=at(2)), ARG),
])
def test_qk_norm_rope(change, expect):
    d = dims()
    args = {**QK, **change, "dims": ctypes.byref(d)}
    assert B.lib().eg_mla_qk_norm_rope(*args.values()) == expect


@pytest.mark.parametrize("change", [
    dict(id_cache=at(6)), dict(id_cache=at(8, 28)), dict(id_cache=at(7)), dict(id_cache=at(9, 128)), dict(id_cache=at(0)),
    dict(id_cache=at(3)), dict(cache=at(4)), dict(cache=at(5, 112)), dict(cache=at(6, 16)), dict(q_out=at(1, 368)),
    dict(q_out=at(7, 16)), dict(q_out=at(10)),
])
def test_qk_norm_rope_outputs_over_weights_and_indices(change):
    d = dims()
    assert B.lib().eg_mla_qk_norm_rope(*{**QK, **change, "dims": ctypes.byref(d)}.values()) == ARG


def test_bad_dims_are_refused_everywhere():
    for kw, expect in [(dict(num_heads=0), ARG), (dict(gate_dim=64), UNSUP), (dict(latent_dim=132), UNSUP)]:
        d = dims(**kw)
        p = ctypes.byref(d)
        L = B.lib()
        assert L.eg_mla_qk_norm_rope(*{**QK, "dims": p}.values()) == expect
        assert L.eg_mla_decode_shared(*{**SHARED, "dims": p}.values()) == expect
        assert L.eg_mla_page_means(*{**MEANS, "dims": p}.values()) == expect
        assert L.eg_mla_page_scores(*{**SCORES, "dims": p}.values()) == expect
        assert L.eg_mla_select_pages(*{**SELECT, "dims": p}.values()) == expect
        assert L.eg_mla_decode_shared_workspace_size(p, 4, 8, 8) == 0
        assert L.eg_mla_page_scores_workspace_size(p, 4) == 0


SHARED = dict(dims=None, batch=4, q=at(0), cache=at(1), ids=at(2), gate=at(3), w_uk=at(4), w_uv=at(5), prefix_len=at(6),
              prefix_table=at(7), prefix_pages=8, lens=at(8), table=at(9), width=8, num_slots=4096, ws=at(10),
              ws_bytes=1 << 30, out=at(11), stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(batch=0), OK), (dict(batch=-1), ARG), (dict(batch=65536), UNSUP), (dict(prefix_pages=-1), ARG), (dict(width=-1), ARG),
    (dict(num_slots=-1), ARG), (dict(num_slots=1 << 31), UNSUP), (dict(num_slots=63), ARG), (dict(width=1 << 25), ARG),
    (dict(prefix_pages=1 << 25), ARG), (dict(q=None), ARG), (dict(cache=None), ARG), (dict(ids=None), ARG),
    (dict(gate=None), ARG), (dict(w_uk=None), ARG), (dict(w_uv=None), ARG), (dict(prefix_len=None), ARG),
    (dict(prefix_table=None), ARG), (dict(lens=None), ARG), (dict(out=None), ARG), (dict(ws=None), WS), (dict(ws_bytes=255), WS),
    (dict(ws=at(10, 16)), WS), (dict(q=at(0, 8)), ARG), (dict(cache=at(1, 8)), ARG), (dict(gate=at(3, 8)), ARG),
    (dict(w_uk=at(4, 8)), ARG), (dict(w_uv=at(5, 8)), ARG), (dict(out=at(11, 8)), ARG),
    (dict(table=None, num_slots=4 * 8 * 64 - 1), ARG),   # contiguous rows that the cache does not hold
])
def test_decode_shared(change, expect):
    d = dims()
    assert B.lib().eg_mla_decode_shared(*{**SHARED, **change, "dims": ctypes.byref(d)}.values()) == expect


@pytest.mark.parametrize("kw", [dict(), dict(latent_dim=320), dict(latent_dim=512, num_heads=128), dict(num_heads=5),
                                dict(dtype=B.FP32, latent_dim=32, rope_dim=0, head_dim=32, v_head_dim=32, num_heads=4)])
def test_decode_shared_workspace_is_enough_and_no_more(kw):
    d = dims(**kw)
    for batch in (1, 3, 64):
        for width, pages in [(0, 0), (8, 0), (0, 300), (16, 300)]:
            n = B.decode_shared_workspace_size(d, batch, width, pages)
            assert n >= 4 * batch * d.num_heads * (d.latent_dim + d.rope_dim) * (1 if n else 0) and n > 0
            if n > 256:
                change = dict(batch=batch, width=width, prefix_pages=pages, ws_bytes=n - 1, num_slots=1 << 20)
                assert B.lib().eg_mla_decode_shared(*{**SHARED, **change, "dims": ctypes.byref(d)}.values()) == WS
    assert B.decode_shared_workspace_size(d, -1, 1, 1) == 0 and B.decode_shared_workspace_size(d, 1, -1, 1) == 0
    assert B.decode_shared_workspace_size(d, 1, 1, -1) == 0 and B.decode_shared_workspace_size(d, 65536, 1, 1) == 0


MEANS = dict(dims=None, batch=4, cache=at(0), ids=at(1), gate=at(2), first=None, lens=at(3), table=at(4), width=8,
             num_slots=1024, means=at(5), stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(batch=0), OK), (dict(width=0), OK), (dict(batch=-1), ARG), (dict(width=-1), ARG), (dict(num_slots=-1), ARG),
    (dict(num_slots=1 << 31), UNSUP), (dict(num_slots=63), ARG), (dict(width=1 << 25), ARG), (dict(cache=None), ARG),
    (dict(ids=None), ARG), (dict(gate=None), ARG), (dict(lens=None), ARG), (dict(means=None), ARG), (dict(cache=at(0, 8)), ARG),
    (dict(gate=at(2, 8)), ARG), (dict(means=at(5, 8)), ARG), (dict(means=at(0, 16)), ARG), (dict(table=None), ARG),
])
def test_page_means(change, expect):
    d = dims()
    assert B.lib().eg_mla_page_means(*{**MEANS, **change, "dims": ctypes.byref(d)}.values()) == expect


SCORES = dict(dims=None, batch=4, q=at(0), w_uk=at(1), means=at(2), lens=at(3), table=at(4), width=8, num_slots=1024, ws=at(5),
              ws_bytes=1 << 20, scores=at(6), stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(batch=0), OK), (dict(width=0), OK), (dict(batch=-1), ARG), (dict(width=-1), ARG), (dict(num_slots=63), ARG),
    (dict(num_slots=1 << 31), UNSUP), (dict(q=None), ARG), (dict(w_uk=None), ARG), (dict(means=None), ARG),
    (dict(lens=None), ARG), (dict(scores=None), ARG), (dict(ws=None), WS), (dict(ws_bytes=4 * 4 * 16 * 192 - 1), WS),
    (dict(ws=at(5, 64)), WS), (dict(q=at(0, 8)), ARG), (dict(w_uk=at(1, 8)), ARG), (dict(means=at(2, 8)), ARG),
    (dict(table=None), ARG),
])
def test_page_scores(change, expect):
    d = dims()
    assert B.lib().eg_mla_page_scores(*{**SCORES, **change, "dims": ctypes.byref(d)}.values()) == expect


SELECT = dict(dims=None, batch=4, scores=at(0), lens=at(1), table=at(2), width=8, keep=5, first=1, last=2, sel=at(3),
              sel_lens=at(4), index=at(5), stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(batch=0), OK), (dict(batch=-1), ARG), (dict(width=-1), ARG), (dict(keep=2), ARG), (dict(first=-1), ARG),
    (dict(last=0), ARG), (dict(width=1 << 25), ARG), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), ARG), (dict(scores=None), ARG),
    (dict(lens=None), ARG), (dict(sel=None), ARG), (dict(sel_lens=None), ARG), (dict(sel=at(2, 4)), ARG),
    (dict(sel_lens=at(1)), ARG), (dict(index=at(3, 8)), ARG), (dict(sel_lens=at(0)), ARG),
    (dict(table=None, batch=1 << 10, width=1 << 22), ARG),
])
def test_select_pages(change, expect):
    d = dims(page_size=16)
    assert B.lib().eg_mla_select_pages(*{**SELECT, **change, "dims": ctypes.byref(d)}.values()) == expect


def test_binding_refuses_tensors_that_are_not_what_the_entry_reads():
    i = torch.int32
    a = lambda *s: torch.zeros(s, dtype=i)  # noqa: E731
    good = [a(2), a(2), a(2, 3), a(9), a(1), a(2), a(3), a(7), a(7), a(1)]
    with pytest.raises(ValueError, match="on cpu"):
        B.page_plan(16, *good)
    with pytest.raises(ValueError, match="on cpu"):
        B.page_release(16, a(2), a(2), a(2, 3), a(9), a(1), a(2), a(1))
    d = dims()
    with pytest.raises(ValueError, match="neither"):
        B.qk_norm_rope(d, None, None, None, None, None, None, None, None)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    with pytest.raises(ValueError, match="q is"):
        B.qk_norm_rope(d, bf(4, 100), bf(4, 16, 192), None, None, None, None, a(4), None)
    with pytest.raises(ValueError, match="kv is"):
        B.qk_norm_rope(d, None, None, bf(4, 384)[:, ::2], bf(9, 192), a(9), a(4), a(4), a(4))
    with pytest.raises(ValueError, match="q_out"):
        B.qk_norm_rope(d, bf(4, 16, 192), bf(3, 16, 192), None, None, None, None, a(4), None)
    with pytest.raises(ValueError, match="on cpu"):
        B.select_pages(d, torch.zeros(2, 3), a(2), a(2, 3), 3, a(2, 2), a(2))
