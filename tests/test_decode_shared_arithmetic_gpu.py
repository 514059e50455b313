"""The arithmetic of eg_mla_decode_shared is that of eg_mla_decode for the layer, whatever the batch."""
import numpy as np
import pytest
import torch

from parity import assert_close, say
from test_decode_shared_gpu import LAYERS, Case

pytestmark = pytest.mark.gpu
LAYERS.update({
    "h5dc128": dict(h=5, dh=128, dv=128, dc=128, dr=64, dtype="bf16"),
    "h20dc320": dict(h=20, dh=128, dv=128, dc=320, dr=64, dtype="bf16"),
    "h3dc512": dict(h=3, dh=128, dv=128, dc=512, dr=64, dtype="bf16"),
    "h12dc128": dict(h=12, dh=64, dv=64, dc=128, dr=64, dtype="bf16"),
    "h12dc320": dict(h=12, dh=64, dv=64, dc=320, dr=64, dtype="bf16"),
    "h8dc512": dict(h=8, dh=64, dv=64, dc=512, dr=64, dtype="bf16"),
})


@pytest.mark.parametrize("layer", ["h5dc128", "h20dc320", "h3dc512", "h12dc128", "h12dc320", "h8dc512"])
@pytest.mark.parametrize("batch", [1, 3, 4, 5, 8, 16])
def test_layers_of_the_fp32_kernels_have_no_16_bit_range(gpu, layer, batch):
    # a gated latent of 10^5 that no head reads: nothing in 32 bits, an infinity in 16
    say(f"decode_shared range {layer} batch={batch}")
    c = Case(layer, 300, [(37 * b) % 90 for b in range(batch)], page=16)
    L = c.L
    L.cache[:, 7], L.gate[:, 7] = 1000.0, 100.0
    L.w_uk[:, :, 7], L.w_uv[:, :, 7] = 0, 0
    assert_close(c.run(), c.ref(), "bf16", layer)
    # nor of an absorbed query: 10^5 times a latent of 2^-17 is a score's ordinary part
    L.cache[:, 7], L.gate[:, 7] = 2.0 ** -17, 1.0
    c.q[:, :, 0], L.w_uk[:, 0, 7] = 512.0, 200.0
    L.w_uk[:, 0, :7] = L.w_uk[:, 0, 8:] = 0
    assert_close(c.run(), c.ref(), "bf16", f"{layer} query")


LAYERS["h128dc128"] = dict(h=128, dh=128, dv=128, dc=128, dr=64, dtype="bf16")


@pytest.mark.parametrize("layer", ["h16", "h48", "h128dc128", "mla320", "h32dc512", "h5dc128", "kv64"])
@pytest.mark.parametrize("prefix,lens", [(200, [40, 0, 130]), (5000, [40, 0, 130]), (700, [4096, 3, 2500])])
def test_partial_rows_keep_what_a_difference_of_latents_leaves(gpu, layer, prefix, lens):
    """Every weight is equal, column 0 holds 1000 or 1004, column 1 1000, and W_UV takes their difference, 4 times a
    fraction: fp16 rows of the prefix's average would be off by up to a quarter each.

    Sums of the values and their count are integers below 2^24, exact in fp32; the average's rounding is 2^-24 of it, and
    as bf16 hi + lo it loses at most 2^-18 of it, 0.0039; the output's own rounding is at most 2^-8 of its size."""
    say(f"decode_shared difference {layer} prefix={prefix} lens={lens}")
    c = Case(layer, prefix, lens)
    L = c.L
    c.q.zero_()
    L.gate.fill_(1)
    L.cache.zero_()
    L.cache[:, 0] = 1000 + 4 * torch.randint(0, 2, (L.cache.shape[0],), generator=L.g).cuda()
    L.cache[:, 1] = 1000
    L.w_uv.zero_()
    L.w_uv[:, :, 0], L.w_uv[:, :, 1] = 1, -1
    got, ref = c.run(), c.ref()
    assert 1 < ref.min() and ref.max() < 3
    off = np.abs(got - ref) - 2.0 ** -8 * np.abs(ref)
    say(f"  {layer}: worst {off.max():.4f}")
    assert off.max() <= 1004 * (2.0 ** -18 + 2.0 ** -22)
