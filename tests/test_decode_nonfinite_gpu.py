"""eg_mla_decode with a NaN among a head's scores: that head's row is not finite, the others are as they are."""
import numpy as np
import pytest
import torch

from paper_2509_16686_amd import binding as B
from parity import assert_close, say
from test_decode_shared_gpu import LAYERS, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layer", sorted(LAYERS))
@pytest.mark.parametrize("lens", [[1], [300, 0, 65], [9000], [3000] * 6, [(91 * b) % 400 + 1 for b in range(40)]], ids=str)
def test_query(gpu, layer, lens):
    say(f"decode NaN query {layer} lens={lens}")
    c = Case(layer, 0, lens)
    L, nb, ref = c.L, len(lens), c.ref()
    c.q[0, 0, 3] = float("nan")
    c.q[nb - 1, L.h - 1, 5] = float("nan")
    ws = B.alloc_workspace(B.decode_workspace_size(L.dims, nb, c.table.shape[1]))
    B.decode(L.dims, c.q, L.cache, L.ids, L.gate, L.w_uk, L.w_uv, c.seq_lens, c.table, c.table.shape[1], ws, c.out)
    torch.cuda.synchronize()
    got, lost = L.f64(c.out), np.zeros((nb, L.h), dtype=bool)
    lost[0, 0] = lost[nb - 1, L.h - 1] = True
    assert np.array_equal(~np.isfinite(got).all(2), lost)
    if not lost.all():
        assert_close(got[~lost], ref[~lost], L.storage, layer)
