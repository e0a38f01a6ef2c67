"""Pin of the cache oracle at the largest magnitudes that its codes hold."""

import numpy as np
import pytest

from oracle import cache_oracle as co


@pytest.mark.parametrize("x,held", [(1.875 * 2.0 ** 127, True), (1.9375 * 2.0 ** 127, False),
                                    (3.3895e38, False), (np.inf, False)])
def test_largest_magnitudes(x, held):
    pool = {"k": np.zeros((1, 1, 64, 96), np.uint8), "v": np.zeros((1, 1, 4, 96, 16), np.uint8),
            "kv_scale": np.ones((1, 1, 2)), "mass": np.zeros((1, 1, 64), np.float32)}
    qkv = np.ones((1, 1, 3, 96))
    qkv[0, 0, 2, 5] = x
    co.append(pool, qkv, np.array([[0]]), [0], [0, 1], 1e4, 1.0)
    k, v, _ = co.tokens(pool, np.array([[0]]), 0, 0, 1)
    assert np.isfinite(k).all() == held
    assert v[0, 5] == (x if held else 0.0)
    assert np.abs(v).max() <= np.finfo(np.float32).max  # every value is one of fp32
