"""RoPE keys that eg_mla_quant_write stores, value by value against those of eg_mla_qk_norm_rope in the bf16 cache."""
import pytest
import torch

from paper_2509_16686_amd import binding as B
from quant_oracle import BF, I32, Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dc,dr", [(128, 64), (512, 64), (48, 24)])
@pytest.mark.parametrize("normed", [False, True])
def test_keys_are_those_of_the_bf16_cache(gpu, dc, dr, normed):
    """Both round the same fp32 rotation once: a value differs by at most one rounding of each (2^-8 of it) and by what the
    two sums of a norm (64 terms: 2^-18) and the two sines and cosines (2^-22) may differ in, relative to its pair."""
    L = Layer(60, 4, 64, 64, dc, dr, rows=256)
    n = 200
    kv, positions, slots = L.normal((n, dc + dr)), L.ints(1 << 20, n), L.perm(256)[:n].contiguous()
    ids, w, kw = L.ints(300, n), L.normal((dc,), 0.1, 1.0), L.normal((dr,), 0.1, 1.0)
    w, kw = (w, kw) if normed else (None, None)
    cache, id_cache = torch.zeros((256, dc + dr), dtype=BF, device="cuda"), torch.zeros(256, dtype=I32, device="cuda")
    B.qk_norm_rope(L.dims, None, None, kv, cache, id_cache, ids, positions, slots, kv_norm_w=w, k_norm_w=kw)
    B.quant_write(L.dims, B.make_rope(), kv, positions, slots, L.codes, L.scales, gate_table=L.gate, token_ids=ids,
                  kv_norm_w=w, k_norm_w=kw)
    a, b = L.codes[slots.long(), dc:].contiguous().view(BF).double(), cache[slots.long(), dc:].double()
    pair = b.reshape(n, dr // 2, 2).abs().sum(2).repeat_interleave(2, 1)
    assert bool(((a - b).abs() <= 2.0 ** -8 * (a.abs() + b.abs()) + 2.0 ** -16 * pair).all())
