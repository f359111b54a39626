"""Helpers of the GPU tests of the 8-bit base, dropout and draft verification, and their error bounds, derived from the
arithmetic.

U is half a step of fp32.  A sum of n products in any order, each exact, is off by at most n U times the sum of their
magnitudes.  The 8-bit matrix instructions keep, of each group of eight products with consecutive k, what lies above
2^-12 of the largest of them: each of the eight loses less than that.  Two bf16 parts of a number are within 2^-17 of it.
Rounding a result to bf16 adds 2^-8 of its value.
"""
import numpy as np

from oracle import dequantize_ref, quantize_ref
from update_helpers import U, f64, out_step, put

E4M3_STEP = 2.0 ** -4


def bytes_of(t):
    """A tensor of 8-bit values or scales as numpy bytes."""
    import torch
    return t.view(torch.uint8).cpu().numpy()


def values_of(t):
    import torch
    return t.view(torch.float8_e4m3fn).cpu().double().numpy()


def rng_of(seed, offset, dev):
    import torch
    return torch.tensor([seed, offset], dtype=torch.int64, device=dev)


def quantized(W, dev):
    """(q, scale, qt, scale_t on the device, their float64 values) of a weight, by the oracle."""
    import torch
    q, e = quantize_ref(W, 128)
    t = torch.tensor(q).to(torch.float8_e4m3fn)
    s = torch.tensor(e + 127).to(torch.uint8)
    return (t.to(dev), s.to(dev), t.t().contiguous().to(dev), s.t().contiguous().to(dev)), dequantize_ref(q, e, 128)


def product_bound(x, W, wide):
    """Bound of x W^T for values x [M, K] and W [N, K] that 8 bits hold: fp32 sums of exact products (wide), or the 8-bit
    instructions."""
    K = x.shape[1]
    tol = K * U * (np.abs(x) @ np.abs(W).T)
    if not wide:
        pad = -K % 8

        def most(a):
            return np.pad(np.abs(a), ((0, 0), (0, pad))).reshape(a.shape[0], -1, 8).max(2)

        tol = tol + 8 * 2.0 ** -12 * (most(x) @ most(W).T)
    return tol


def linear_bounds(x, W, A, B, s, y_type, xa=None):
    """Bounds of y_off and y_on; x: the values after quantizing, W the weight's, xa the adapter's input."""
    M, K = x.shape
    wide = M <= 16 or y_type == "f32"
    off = product_bound(x, W, wide)
    on = off.copy()
    if A is not None and len(A):
        r = len(A)
        t = np.abs(xa) @ np.abs(A).T
        # T's sum and its product with s, two parts of it above 16 rows, the products with B and their sum
        on = on + abs(s) * (((K + 2) * U + (2.0 ** -17 if M > 16 else 0) + (2 * r + 2) * U) * (t @ np.abs(B).T))
    return off, on


def rounded(tol, ref, y_type):
    """The bound of an output of this type from that of its value."""
    return tol + out_step(y_type) * (np.abs(ref) + tol) + 1e-40


def backward_bounds(xa, W, A, B, s, dy, dx_type, factor):
    """Bounds of dx, dA, dB (W [N, K]: the weight's values)."""
    M, N = dy.shape
    K, r = W.shape[1], len(A)
    dq = dequantize_ref(*quantize_ref(dy, 1), 1)
    wide = dx_type == "f32"
    u = abs(s) * (np.abs(dy) @ np.abs(B))
    t = abs(s) * (np.abs(xa) @ np.abs(A).T)
    # (dx takes two bf16 parts of s U, dA and dB three, which are within 2^-25 of it)
    r_u, r_t = (N + 2.5) * U, (K + 2.5) * U
    dx = product_bound(dq, W.T, wide) + (r_u + 2.0 ** -17 + (2 * r + 4) * U) * (u @ np.abs(A)) * np.maximum(factor, 0)
    dA = (r_u + (3 * M + 2) * U) * (u.T @ np.abs(xa))
    dB = (r_t + (3 * M + 2) * U) * (np.abs(dy).T @ t)
    return dx, dA + 1e-40, dB + 1e-40
