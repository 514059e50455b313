"""Calls of the row rotation and the 8-bit cache that are refused on the host, before anything is enqueued: by the C
entries (pointers that nothing reads) and by the binding (tensors that the entries would misread)."""
import ctypes
import math

import pytest
import torch

from paper_2509_16686_amd import binding as B

OK, ARG, UNSUP, WS = B.OK, B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED, B.ERR_WORKSPACE
BIG = 1 << 28  # made-up addresses, 256 MiB apart


def at(i, off=0):
    return ctypes.c_void_p(BIG * (i + 1) + off)


def dims(**kw):
    base = dict(num_heads=16, head_dim=128, v_head_dim=128, latent_dim=128, rope_dim=64, vocab_size=500, page_size=64)
    base.update(kw)
    return B.make_dims(**base)


def rope(**kw):
    return B.make_rope(**kw)


# 8 tokens of 4 heads of 192 values, the last 64 rotated
ROPE = dict(rope=None, dtype=B.BF16, n=8, heads=4, dim=192, off=128, rd=64, x=at(0), xt=768, xh=192, positions=at(1), inverse=0,
            out=at(2), ot=768, oh=192, stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(n=0), OK), (dict(n=0, x=None), OK), (dict(n=-1), ARG), (dict(heads=0), ARG), (dict(dim=0), ARG), (dict(dtype=7), ARG),
    (dict(rd=63), ARG), (dict(rd=-2), ARG), (dict(off=-1), ARG), (dict(off=129), ARG), (dict(dim=100), ARG),
    (dict(off=2 ** 31 - 1), ARG), (dict(dim=700, rd=642, off=0, xt=2800, xh=700, ot=2800, oh=700), UNSUP),
    (dict(x=None), ARG), (dict(out=None), ARG), (dict(positions=None), ARG), (dict(x=at(0, 1)), ARG), (dict(out=at(2, 1)), ARG),
    (dict(dtype=B.FP32, x=at(0, 2)), ARG), (dict(xt=-1), ARG), (dict(xh=-192), ARG), (dict(ot=(1 << 32) + 8), ARG),
    (dict(ot=0), ARG), (dict(oh=0), ARG), (dict(oh=191), ARG), (dict(ot=767), ARG), (dict(ot=100, oh=191), ARG),
    (dict(out=at(0), ot=776), ARG), (dict(out=at(0, 384)), ARG), (dict(out=at(1)), ARG), (dict(out=at(1, 16)), ARG),
    (dict(rope=rope(layout=2)), ARG), (dict(rope=rope(theta=math.inf)), ARG), (dict(rope=rope(theta=math.nan)), ARG),
    (dict(rope=rope(magnitude=math.inf)), ARG), (dict(rope=rope(magnitude=math.nan)), ARG),
    (dict(rope=rope(frequencies=[1.0] * 31 + [math.nan])), ARG), (dict(rope=rope(frequencies=[math.inf] + [1.0] * 31)), ARG),
    (dict(rope=rope(frequencies=[-64.5] + [1.0] * 31)), ARG),
])
def test_rope_rows(change, expect):
    args = {**ROPE, "rope": rope(), **change}
    args["rope"] = ctypes.byref(args["rope"])
    assert B.lib().eg_mla_rope_rows(*args.values()) == expect


def test_rope_rows_needs_a_rotation():
    assert B.lib().eg_mla_rope_rows(*ROPE.values()) == ARG


@pytest.mark.parametrize("change,expect", [
    (dict(), OK), (dict(factor=1.0), OK), (dict(trained=0), OK), (dict(theta=0.0), OK), (dict(rd=0), ARG), (dict(rd=63), ARG),
    (dict(rd=642), ARG), (dict(factor=0.5), ARG), (dict(factor=math.inf), ARG), (dict(factor=math.nan), ARG),
    (dict(theta=math.nan), ARG), (dict(theta=math.inf), ARG), (dict(trained=-1), ARG), (dict(slow=32.0), ARG),
    (dict(slow=5.0, fast=4.0), ARG), (dict(out=None), ARG),
])
def test_rope_frequencies(change, expect):
    base = dict(rd=64, theta=10000.0, factor=4.0, trained=4096, slow=0.0, fast=0.0, out=(ctypes.c_double * 321)())
    assert B.lib().eg_mla_rope_frequencies(*{**base, **change}.values()) == expect


@pytest.mark.parametrize("change,size", [
    (dict(), 256), (dict(latent_dim=512), 640), (dict(latent_dim=48, rope_dim=24), 96), (dict(rope_dim=0), 128),
    (dict(latent_dim=120), 0), (dict(latent_dim=528), 0), (dict(rope_dim=72), 0), (dict(dtype=B.FP32), 0), (dict(num_heads=0), 0),
])
def test_row_bytes(change, size):
    assert B.quant_row_bytes(dims(**change)) == size


WRITE = dict(dims=None, rope=None, n=8, kv=at(0), stride=192, kv_w=at(1), k_w=at(2), gate=at(3), ids=at(4), positions=at(5),
             slots=at(6), codes=at(7), scales=at(8), num_slots=1024, stream=None)


@pytest.mark.parametrize("layer,change,expect", [
    ({}, dict(n=0, kv=None), OK), ({}, dict(n=-1), ARG), ({}, dict(num_slots=-1), ARG), (dict(dtype=B.FP32), {}, UNSUP),
    (dict(latent_dim=136), {}, UNSUP), (dict(rope_dim=72), dict(stride=200), UNSUP), (dict(latent_dim=528), dict(stride=592), UNSUP),
    ({}, dict(kv=None), ARG), ({}, dict(slots=None), ARG), ({}, dict(codes=None), ARG), ({}, dict(scales=None), ARG),
    ({}, dict(ids=None), ARG), ({}, dict(positions=None), ARG), ({}, dict(stride=184), ARG), ({}, dict(stride=196), ARG),
    ({}, dict(stride=(1 << 32) + 8), ARG), ({}, dict(kv=at(0, 8)), ARG), ({}, dict(gate=at(3, 8)), ARG),
    ({}, dict(kv_w=at(1, 8)), ARG), ({}, dict(codes=at(7, 8)), ARG),
    ({}, dict(codes=at(0)), ARG), ({}, dict(codes=at(8)), ARG), ({}, dict(scales=at(6)), ARG), ({}, dict(scales=at(5, 31)), ARG),
    ({}, dict(scales=at(4)), ARG), ({}, dict(codes=at(3)), ARG), ({}, dict(scales=at(2, 127)), ARG), ({}, dict(codes=at(1)), ARG),
    ({}, dict(scales=at(7, 1024 * 256 - 1)), ARG), ({}, dict(rope=rope(layout=-1)), ARG),
])
def test_write(layer, change, expect):
    args = {**WRITE, "rope": rope(), **change}
    args["dims"], args["rope"] = ctypes.byref(dims(**layer)), ctypes.byref(args["rope"])
    assert B.lib().eg_mla_quant_write(*args.values()) == expect


READ = dict(dims=None, batch=4, total=100, codes=at(0), scales=at(1), first=at(2), cu=at(3), table=at(4), pages=8,
            num_slots=1024, out=at(5), stream=None)


@pytest.mark.parametrize("layer,change,expect", [
    ({}, dict(batch=0), OK), ({}, dict(total=0), OK), ({}, dict(pages=0), OK), ({}, dict(batch=-1), ARG),
    ({}, dict(batch=4097), UNSUP), ({}, dict(total=-1), ARG), ({}, dict(pages=-1), ARG), ({}, dict(pages=1 << 25), ARG),
    ({}, dict(table=None), ARG), ({}, dict(num_slots=63), ARG), ({}, dict(num_slots=1 << 31), UNSUP),
    (dict(dtype=B.FP32), {}, UNSUP), ({}, dict(codes=None), ARG), ({}, dict(scales=None), ARG), ({}, dict(cu=None), ARG),
    ({}, dict(out=None), ARG), ({}, dict(codes=at(0, 8)), ARG), ({}, dict(out=at(5, 8)), ARG), ({}, dict(out=at(0)), ARG),
    ({}, dict(out=at(1)), ARG), ({}, dict(out=at(2)), ARG), ({}, dict(out=at(3, 16)), ARG), ({}, dict(out=at(4, 112)), ARG),
])
def test_read(layer, change, expect):
    args = {**READ, **change}
    args["dims"] = ctypes.byref(dims(**layer))
    assert B.lib().eg_mla_quant_read(*args.values()) == expect


ATTEND = dict(dims=None, batch=4, n=4, q=at(0), cu=at(1), codes=at(2), scales=at(3), w_uk=at(4), w_uv=at(5), lens=at(6),
              table=at(7), pages=8, num_slots=1024, ws=at(10), ws_bytes=1 << 28, out=at(8), stream=None)


@pytest.mark.parametrize("layer,change,expect", [
    ({}, dict(batch=0, n=0), OK), ({}, dict(n=0), OK), ({}, dict(batch=-1), ARG), ({}, dict(n=-1), ARG),
    ({}, dict(batch=4097), UNSUP), ({}, dict(n=(1 << 19) + 1), UNSUP), (dict(num_heads=1 << 12), dict(n=1 << 19), UNSUP), (dict(num_heads=1 << 23), {}, UNSUP),
    (dict(), dict(n=1 << 19, pages=1 << 24, num_slots=1 << 20), UNSUP),
    ({}, dict(pages=-1), ARG), ({}, dict(pages=1 << 25), ARG), ({}, dict(cu=None, n=5), ARG), ({}, dict(table=None), ARG),
    ({}, dict(num_slots=63), ARG), ({}, dict(num_slots=1 << 31), UNSUP), (dict(dtype=B.FP32), {}, UNSUP),
    (dict(latent_dim=136), {}, UNSUP), (dict(rope_dim=72), {}, UNSUP),
    ({}, dict(q=None), ARG), ({}, dict(codes=None), ARG), ({}, dict(scales=None), ARG), ({}, dict(w_uk=None), ARG),
    ({}, dict(w_uv=None), ARG), ({}, dict(lens=None), ARG), ({}, dict(out=None), ARG), ({}, dict(q=at(0, 8)), ARG),
    ({}, dict(codes=at(2, 8)), ARG), ({}, dict(w_uk=at(4, 8)), ARG), ({}, dict(w_uv=at(5, 8)), ARG), ({}, dict(out=at(8, 8)), ARG),
    ({}, dict(ws=None), WS), ({}, dict(ws=at(10, 16)), WS), ({}, dict(ws_bytes=1000), WS),
    ({}, dict(out=at(0)), ARG), ({}, dict(out=at(1)), ARG), ({}, dict(out=at(2)), ARG), ({}, dict(out=at(3)), ARG),
    ({}, dict(out=at(4)), ARG), ({}, dict(out=at(5)), ARG), ({}, dict(out=at(6)), ARG), ({}, dict(out=at(7)), ARG),
    ({}, dict(out=at(10)), ARG), ({}, dict(q=at(10)), ARG), ({}, dict(scales=at(10)), ARG), ({}, dict(lens=at(10)), ARG),
])
def test_attend(layer, change, expect):
    args = {**ATTEND, **change}
    args["dims"] = ctypes.byref(dims(**layer))
    assert B.lib().eg_mla_quant_attend(*args.values()) == expect


def test_workspace_size():
    d = dims()
    assert B.quant_attend_workspace_size(dims(dtype=B.FP32), 4, 4, 8) == 0
    assert B.quant_attend_workspace_size(d, 4097, 4097, 8) == 0
    assert B.quant_attend_workspace_size(d, -1, 4, 8) == 0
    assert B.quant_attend_workspace_size(d, 4, 4, 1 << 25) == 0


@pytest.mark.parametrize("heads,dc", [(1, 48), (12, 64), (16, 128), (20, 320), (128, 512), (24, 512)])
def test_workspace_of_the_largest_call_serves_smaller_ones(heads, dc):
    d = dims(num_heads=heads, latent_dim=dc)
    sizes = [(b, n, p) for b in (1, 3, 16, 200, 4096) for n in (1, 7, 64, 300, 5000) for p in (1, 8, 500)]
    held = {s: B.quant_attend_workspace_size(d, *s) for s in sizes}
    assert all(v % 256 == 0 and v > 0 for v in held.values())
    for s in sizes:
        for big in sizes:
            if all(x <= y for x, y in zip(s, big)):
                assert held[s] <= held[big], (s, big)


def _cpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_refuses():
    d, i32, u8 = dims(), torch.int32, torch.uint8
    codes, scales, slots = _cpu(64, 256, dtype=u8), _cpu(64, dtype=u8), _cpu(8, dtype=i32)
    kv, x = _cpu(8, 192), _cpu(8, 4, 192)
    bad = [
        lambda: B.rope_rows(rope(), x, slots, x, rope_dim=64),                        # on the host
        lambda: B.rope_rows(rope(frequencies=[1.0] * 3), x, slots, x, rope_dim=64),
        lambda: B.rope_rows(rope(), x.half(), slots, x.half(), rope_dim=64),
        lambda: B.rope_rows(rope(), x, slots, x.float(), rope_dim=64),
        lambda: B.rope_rows(rope(), x.transpose(1, 2), slots, x.transpose(1, 2), rope_dim=2),
        lambda: B.quant_write(d, rope(), kv, slots, slots, codes, scales),
        lambda: B.quant_write(d, rope(), kv.float(), slots, slots, codes, scales),
        lambda: B.quant_write(d, rope(), kv[:, :100], slots, slots, codes, scales),
        lambda: B.quant_read(d, codes, scales, None, slots, None, kv),
        lambda: B.quant_read(d, codes, scales, None, slots, slots.reshape(2, 4), kv),
        lambda: B.quant_attend(d, _cpu(8, 16, 192), None, codes, scales, _cpu(16, 128, 128), _cpu(16, 128, 128), slots,
                            slots.reshape(8, 1), 1, _cpu(1000, dtype=u8), _cpu(8, 16, 128)),
    ]
    for call in bad:
        with pytest.raises((ValueError, B.EgMlaError)):
            call()
