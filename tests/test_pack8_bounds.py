"""How far the coding in 8 bits may move a value, as include/sdnn.h states it: over all exponents, in the plain form that the kernels' bytes are compared with."""
import numpy as np
import pytest

from tests import blocks

TOP = np.finfo(np.float32).max


def groups(seed):
    """Groups of 128 values up to a largest one: every power of two, numbers between, the ends of the floats."""
    rng = np.random.default_rng(seed)
    largest = np.concatenate([2.0 ** np.arange(-149, 128), 1.999 * 2.0 ** np.arange(-148, 128), 127 * 2.0 ** np.arange(-149.0, 121), 253 * 2.0 ** np.arange(-149.0, 120),
                              [1e-44, 3.4e38, 3.40262e38, 3.4027e38, TOP, np.nextafter(TOP, np.float32(0))]])
    x = largest[:, None] * rng.uniform(-1, 1, (largest.size, 128))
    x[:, 5], x[:, 6] = largest, -largest
    return x.astype(np.float32)


@pytest.mark.parametrize("cap", [0.0, 1.0, float("inf")])
def test_bounds_of_scales_and_values(cap):
    x = groups(1)
    codes, scales, value = blocks.pack8(x, cap)
    t = (scales.astype(np.uint32) << 16).view(np.float32).astype(np.float64)[:, None]
    v = np.clip(x.astype(np.float64), 0, cap) if cap > 0 else x.astype(np.float64)
    most = 253 if cap > 0 else 127
    largest = np.where((v < cap) | (cap == 0), np.abs(v), 0).max(1, keepdims=True)
    assert np.all(most * t >= largest) and np.all(t <= 1.008 * largest / most + 2.0 ** -133)
    low = (v < t / 2) & (cap > 0)
    assert np.all(np.abs(value - v) <= np.where(low, t, t / 2))
    with np.errstate(over="ignore"):
        assert np.isfinite(value.astype(np.float32)).all()
    if cap == 0:  # the product that brings a code back, in fp32
        product = codes.view(np.int8).reshape(x.shape).astype(np.float32) * t.astype(np.float32)
        assert np.isfinite(product).all() and np.array_equal(product, value)
