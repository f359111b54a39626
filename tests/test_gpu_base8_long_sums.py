"""The 8-bit base at the largest K, on numbers whose sums are exact: whole numbers of at most 2, so that a sum of 2^21 products
stays below 2^24 in every order, each block of K times a power of two of its own in x and its inverse in W, each row of x
times one of its own.  Quantization, products, parts of K and their joining change nothing then: fp32 outputs have to have
the sum's bits, bf16 ones its nearest value's.  The adapter has few entries, at both ends of K and of its blocks, so that
T is exact too."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from gpu_helpers import say
from update_helpers import dtype, empty, f64

pytestmark = pytest.mark.gpu

LONGEST = 1 << 21


@pytest.fixture(autouse=True)
def leave_no_memory():
    import torch
    yield
    torch.cuda.empty_cache()


class Whole:
    """rows [M, K] and weight [N, K] of whole numbers, `turn` the blocks' powers; adapter rows [r, K] and columns [N, r]."""

    def __init__(self, seed, M, N, K, r, dev):
        g = np.random.default_rng(seed)
        self.dev = dev
        kb = -(-K // 128)
        self.x = g.integers(-2, 3, (M, K)).astype(np.float32)
        self.w = g.integers(-2, 3, (N, K)).astype(np.float32)
        self.block = np.repeat(g.integers(-20, 21, kb), 128)[:K]
        self.row = g.integers(-2, 3, M)
        at = np.unique(np.r_[0, 1, 127, 128, K // 2 - 1, K // 2, K - 129, K - 128, K - 1, g.integers(0, K, 20)])
        self.A = np.zeros((r, K), np.float32)
        self.A[:, at] = g.integers(-2, 3, (r, len(at)))
        self.B = g.integers(-2, 3, (N, r)).astype(np.float32)

    def bf16(self, a, block=0, row=None):
        import torch
        a = np.ldexp(a, self.block * block) if block else a
        return torch.as_tensor(np.ldexp(a, row[:, None]) if row is not None else a).to(self.dev).bfloat16()

    def quantized(self, w, transposed=False):
        import torch
        N, K = w.shape

        def room(*shape):
            return torch.empty(shape, dtype=torch.uint8, device=self.dev)

        q, s, qt, st = room(N, K), room(-(-N // 128), -(-K // 128)), None, None
        if transposed:
            qt, st = room(K, N), room(-(-K // 128), -(-N // 128))
        H.hydra_fp8_quantize(w, q, s, 128, qt, st)
        return (qt, st) if transposed else (q, s)


def nearest(v, y_type):
    import torch
    assert np.abs(v).max() > 0
    return torch.as_tensor(v).to(dtype(y_type)).double().numpy()


@pytest.mark.parametrize("M,N", [(2, 5), (16, 40), (17, 5), (40, 200), (130, 70)])
@pytest.mark.parametrize("K", [LONGEST, LONGEST - 16])
def test_the_longest_sums(dev, M, N, K):
    say("longest sums", M, N, K)
    c = Whole(M + N, M, N, K, 3, dev)
    x, A, B = c.bf16(c.x, 1, c.row), c.bf16(c.A, -1), c.bf16(c.B)
    q, s = c.quantized(c.bf16(c.w, -1))
    off = np.ldexp((c.x @ c.w.T).astype(np.float64), c.row[:, None])
    on = off + np.ldexp(2.0 * ((c.x @ c.A.T) @ c.B.T).astype(np.float64), c.row[:, None])
    for y_type in ("f32", "bf16"):
        y = [empty((M, N), y_type, dev) for _ in range(2)]
        H.hydra_fp8_lora_linear(x, q, s, A, B, 2.0, *y)
        for g, e, name in zip(y, (off, on), ("y_off", "y_on")):
            assert np.array_equal(f64(g), nearest(e, y_type)), f"{name} {y_type}"


@pytest.mark.parametrize("M,K", [(3, 16), (40, 48), (70, 144)])
def test_the_longest_sums_of_the_backward(dev, M, K):
    """dx sums over N outputs: dy takes x's place, the weight's transpose W's."""
    say("longest sums of the backward", M, K)
    c = Whole(M + K, M, K, LONGEST, 2, dev)      # (its x: dy; its w: the weight's transpose; its A: B^T; its B: A^T)
    dy, B, A = c.bf16(c.x, 1, c.row), c.bf16(c.A, -1).t().contiguous(), c.bf16(c.B).t().contiguous()
    qt, st = c.quantized(c.bf16(c.w, -1).t().contiguous(), transposed=True)
    xa = np.random.default_rng(1).integers(-2, 3, (M, K)).astype(np.float32)
    dx = np.ldexp((c.x @ c.w.T + 2.0 * (c.x @ c.A.T) @ c.B.T).astype(np.float64), c.row[:, None])
    u = np.ldexp(2.0 * (c.x @ c.A.T).astype(np.float64), c.row[:, None])
    for t in ("f32", "bf16"):
        got = empty((M, K), t, dev)
        dA, dB = empty((2, K), "f32", dev), empty((LONGEST, 2), "f32", dev)
        H.hydra_fp8_lora_linear_backward(c.bf16(xa), qt, st, A, B, 2.0, dy, got, dA, dB)
        assert np.array_equal(f64(got), nearest(dx, t)), f"dx {t}"
        assert np.array_equal(f64(dA), u.T @ xa), "dA"
        at = np.r_[0:300, LONGEST // 2:LONGEST // 2 + 300, LONGEST - 300:LONGEST]
        d = np.ldexp(np.ldexp(c.x[:, at], c.block[at]), c.row[:, None]).astype(np.float64)
        assert np.array_equal(f64(dB[at.tolist()]), 2.0 * d.T @ (xa @ c.B).astype(np.float64)), "dB"
