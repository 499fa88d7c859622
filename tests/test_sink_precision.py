"""The limit that test_gpu_sink_precision.py holds the kernels to tells three bf16 parts from two."""
import numpy as np
import pytest

import oracle as O

from sink_precision import LIMIT, error, modelled


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("T", [90, 700])
def test_the_limit_tells_three_parts_from_two(hd, T):
    rng = np.random.default_rng(hd + T)
    k, v = (O.mx_values(*O.mx_round(rng.standard_normal((T, hd)))) for _ in range(2))
    q = rng.standard_normal((32, hd)).astype(np.float32)
    s = q.astype(np.float64) @ k.T / np.sqrt(hd)
    w = np.exp(s - s.max(1, keepdims=True))
    ref = w @ v / w.sum(1, keepdims=True)
    assert error(modelled(q, k, v, 3, 3), ref) < LIMIT / 2
    assert error(modelled(q, k, v, 2, 3), ref) > 4 * LIMIT
    assert error(modelled(q, k, v, 3, 2), ref) > 1.25 * LIMIT
    assert error(modelled(q, k, v, 3, 1), ref) > 500 * LIMIT
