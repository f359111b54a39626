"""How many bits of s T (s U) the update over an 8-bit base takes into fp32 outputs: all that fp32 holds.  T and U are exact here
(whole numbers, few of them), the weight is zero, and s has 24 bits, so that an output is a sum of a few products of a
24-bit number and a bf16 one.  Sizes of every tile, whole and in parts of K, with few and many partial sums of T, with and
without dropout's mask."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from base8_helpers import rng_of
from gpu_helpers import say
from update_helpers import U, empty, f64, near, put

pytestmark = pytest.mark.gpu

S = float(np.float32(1.2345678))


def whole(g, M, K, r, dev):
    """rows [M, K] and adapter rows [r, K] in bf16, and T = rows adapter^T: at most three of the r rows are not zero, and
    few entries of those."""
    x = g.integers(-3, 4, (M, K)).astype(np.float32)
    A = np.zeros((r, K), np.float32)
    at = np.unique(g.integers(0, K, 24))
    for j in {0, r // 2, r - 1}:
        A[j, at] = g.integers(-3, 4, len(at))
    return put(x, "bf16", dev), put(A, "bf16", dev), (x @ A.T).astype(np.float64)


def update(T, B):
    """s T B^T and its bound: s T rounded once, each of its three parts times B exact, their sum."""
    t, b = np.float64(S) * T, np.abs(B).T
    return t @ B.T, 12 * U * (np.abs(t) @ b) + 1e-40


@pytest.mark.parametrize("M,N,K,r", [
    (5, 100, 256, 3), (17, 64, 128, 1), (40, 300, 1024, 4), (64, 4096, 528, 16), (333, 264, 2064, 16), (130, 8200, 128, 20),
    (1100, 2052, 272, 100), (2050, 2600, 128, 16), (17, 2048, 8192, 16), (300, 40, 16000, 128), (64, 514, 8208, 3),
    (653, 1966, 8192, 2), (333, 4096, 11008, 16),
])
def test_update_of_the_forward(dev, M, N, K, r):
    import torch
    say("bits of the update", M, N, K, r)
    g = np.random.default_rng(M + K)
    x, A, T = whole(g, M, K, r, dev)
    B = put(g.normal(0, 0.3, (N, r)), "bf16", dev)
    W, w = torch.zeros((N, K), dtype=torch.uint8, device=dev), torch.full((-(-N // 128), -(-K // 128)), 127, dtype=torch.uint8, device=dev)
    off, on = empty((M, N), "f32", dev), empty((M, N), "f32", dev)
    H.hydra_fp8_lora_linear(x, W, w, A, B, S, off, on)
    ref, tol = update(T, f64(B))
    assert (off == 0).all()
    near(f64(on), ref, tol, "y_on")


@pytest.mark.parametrize("M,N,K,r", [(3, 64, 48, 8), (40, 144, 400, 5), (130, 528, 256, 64), (1030, 256, 2064, 16),
                                     (1100, 144, 2608, 16), (2050, 64, 2608, 128), (64, 4112, 144, 128), (250, 8192, 1040, 128)])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_update_of_the_backward(dev, M, N, K, r, p):
    import torch
    say("bits of the backward's update", M, N, K, r, p)
    g = np.random.default_rng(M + N)
    dy, B, T = whole(g, M, N, r, dev)
    A = put(g.normal(0, 0.3, (r, K)), "bf16", dev)
    W, w = torch.zeros((K, N), dtype=torch.uint8, device=dev), torch.full((-(-K // 128), -(-N // 128)), 127, dtype=torch.uint8, device=dev)
    dx, mask, rng = empty((M, K), "f32", dev), empty((M, K), "f32", dev), rng_of(9, 4, dev)
    H.hydra_fp8_lora_linear_backward(None, W, w, A, B.t().contiguous(), S, dy, dx, p=p, rng=rng)
    H.hydra_dropout(torch.ones((M, K), device=dev), mask, p, rng)  # (pinned element by element in the tests of dropout)
    ref, tol = update(T, f64(A).T)
    near(f64(dx), ref * f64(mask), (tol + 3 * U * np.abs(ref)) * f64(mask) + 1e-40, "dx")
