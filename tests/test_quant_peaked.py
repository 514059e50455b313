"""The bound of the peaked attention cases (quant_peaked.py) is tight enough to see one tile or 8 values of one key."""
import numpy as np
import pytest

from quant_peaked import Peaked

SHAPES = {64: (12, 64, 64, 64, 64), 128: (16, 128, 128, 128, 64), 144: (16, 64, 136, 144, 64), 320: (16, 128, 128, 320, 64),
          512: (16, 128, 128, 512, 64)}


@pytest.mark.parametrize("dc", SHAPES)
@pytest.mark.parametrize("peaks", ["rope", "latent"])
def test_one_tile_or_8_values_of_one_key_exceed_the_bound(dc, peaks):
    P = Peaked(dc, *SHAPES[dc], [11], [1500], peaks, 32)
    want, bound = P.attend()
    other = Peaked(dc + 1, *SHAPES[dc], [11], [1500], peaks, 32)

    def tile(t):
        def change(b, lat, p):
            p[:, 32 * t: 32 * t + 32] = 0
            return lat, p
        return change

    def key(t):
        def change(b, lat, p):  # (of the next key's magnitude)
            lat[32 * t, :8] = other.lat[b][32 * t, :8] * np.abs(lat[32 * t]).max() / np.abs(other.lat[b][32 * t]).max()
            return lat, p
        return change

    seen = [[(np.abs(P.attend(f(t))[0] - want) / bound).max() > 1 for t in range(1, 46, 4)] for f in (tile, key)]
    assert np.mean(seen[0]) == 1 and np.mean(seen[1]) >= (0.9 if peaks == "rope" else 0.4), [np.mean(x) for x in seen]
