"""Sizes whose bytes pass 64 bits still meet the arrays behind them (host checks; pointers that nothing reads)."""
import ctypes

import pytest

from paper_2509_16686_amd import binding as B
from test_server_refusals import QK, SCORES, SELECT, dims

INT_MAX = 2 ** 31 - 1


def far(args):
    """The call's made-up addresses, 2^46 bytes apart."""
    at = 0
    out = {}
    for k, v in args.items():
        if isinstance(v, ctypes.c_void_p):
            at += 1
            v = ctypes.c_void_p(at << 46)
        out[k] = v
    return out


@pytest.mark.parametrize("change", [
    dict(n=INT_MAX, q_stride=1 << 32, kv=None),               # q's rows reach q_out
    dict(n=INT_MAX, kv_stride=1 << 32, q=None, num_slots=1),  # kv's the cache
    dict(num_slots=1 << 62),                                  # the cache the ids' cache
])
def test_qk_norm_rope(change):
    d = dims(dtype=B.FP32)
    assert B.lib().eg_mla_qk_norm_rope(*{**far(QK), **change, "dims": ctypes.byref(d)}.values()) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("change", [
    dict(batch=INT_MAX, keep=INT_MAX, width=1, index=None),       # the choice reaches the lengths written
    dict(batch=INT_MAX, width=1 << 26, keep=4, index=None),       # the scores reach the choice
])
def test_select_pages(change):
    d = dims(page_size=16)
    assert B.lib().eg_mla_select_pages(*{**far(SELECT), **change, "dims": ctypes.byref(d)}.values()) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(), dict(dtype=B.FP32), dict(head_dim=32)])
def test_page_scores(kw):
    d = dims(num_heads=1 << 30, latent_dim=512, **kw)
    assert B.page_scores_workspace_size(d, 1 << 30) >= 2 ** 63 - 1
    args = {**far(SCORES), "batch": 1 << 30, "dims": ctypes.byref(d)}
    assert B.lib().eg_mla_page_scores(*args.values()) == B.ERR_WORKSPACE
