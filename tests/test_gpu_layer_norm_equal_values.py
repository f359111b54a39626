"""Rows of one value: the mean of K equal values is that value, whatever K.

The sums of these rows are exact in fp32 in any order (whole numbers, or quarters, below 2^24 of their unit), so a mean
that divides the sum by K is exact, the centred values are 0 and the result is the bias bit for bit; the backward's two
means leave a gradient of exactly 0.  A mean formed with the rounded 1 / K misses the value by a step at thousands of
the widths up to 16384."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from gpu_helpers import say
from update_helpers import TYPES, empty, f64, put

pytestmark = pytest.mark.gpu

# of 1 to 16 waves a row, with and without 16-byte groups, and rows past what the registers hold
WIDTHS = [1, 7, 15, 56, 60, 75, 120, 255, 1000, 1001, 2047, 2048, 3736, 4099, 5880, 8191, 8560, 9445, 9824, 11008, 13039,
          16383, 16384, 16386]
VALUES = np.array([1000.0, 7.0, 3.25, -10.0, 3.0, -0.75, 0.0, 240.0])


@pytest.mark.parametrize("y_type", TYPES)
@pytest.mark.parametrize("x_type", TYPES)
def test_the_result_is_the_bias(x_type, y_type, dev):
    for K in WIDTHS:
        for shift in (0, 1):
            say("equal values", K, x_type, y_type, shift)
            x = np.repeat(VALUES[:, None], K, 1)
            assert (np.abs(VALUES) * K < 2 ** 24).all()
            w, b = (put(v, y_type, dev, shift) for v in np.random.default_rng(K).normal(0, 1, (2, K)))
            M = len(VALUES)
            y, mean, rstd = empty((M, K), y_type, dev, shift), empty(M, "f32", dev), empty(M, "f32", dev)
            H.hydra_layer_norm(put(x, x_type, dev, shift), w, b, y, mean, rstd, eps=0.25)
            assert np.array_equal(f64(mean), VALUES), (K, shift, f64(mean))
            assert (f64(rstd) == 2).all(), (K, shift)
            assert np.array_equal(f64(y), np.repeat(f64(b)[None], M, 0)), (K, shift)


@pytest.mark.parametrize("dy_type", TYPES)
@pytest.mark.parametrize("x_type", TYPES)
def test_an_equal_gradient_passes_nothing_on(dy_type, x_type, dev):
    M = len(VALUES)
    for K in WIDTHS:
        for shift in (0, 1):
            say("equal gradients", K, dy_type, x_type, shift)
            rows = put(np.repeat(VALUES[:, None], K, 1), dy_type, dev, shift)
            x = put(np.full((M, K), 5.0), x_type, dev, shift)
            mean, rstd = put(np.full(M, 5.0), "f32", dev), put(np.full(M, 2.0), "f32", dev)
            dx = empty((M, K), "f32", dev, shift)
            H.hydra_layer_norm_backward(rows, x, None, mean, rstd, dx)
            assert (f64(dx) == 0).all(), (K, shift)
