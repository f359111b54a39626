"""The linear over an 8-bit base and its backward in a workspace of exactly the promised size: what lies behind it stays as it
is, and no stage's operands are overwritten by another's sums.  Sizes where K is taken in parts, among them those with more
than 256 parts of 128 x 256 outputs."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import dequantize_ref, fp8_linear_backward_ref, fp8_linear_ref, quantize_ref
from base8_helpers import backward_bounds, f64, linear_bounds, rng_of, rounded
from gpu_helpers import say
from test_gpu_fp8_linear import S, Linear
from update_helpers import U, empty, near

pytestmark = pytest.mark.gpu

GUARD, BYTE = 64 << 20, 0xA5


def guarded(n, dev):
    import torch
    flat = torch.full((n + GUARD,), BYTE, dtype=torch.uint8, device=dev)
    return flat[:n], flat[n:]


def some(M):
    """Rows of every tile, and the last ones (few rows: all)."""
    return np.arange(M) if M <= 300 else np.unique(np.r_[np.arange(0, M, 9), np.arange(M - 5, M)])


@pytest.mark.parametrize("M,N,K,r,y_type", [
    (1280, 4096, 11008, 16, "f32"), (2100, 2048, 8192, 20, "f32"), (3585, 1030, 12288, 16, "bf16"),
    (1050, 4096, 8192, 128, "f32"), (333, 4096, 11008, 16, "f32"), (17, 2048, 8192, 16, "bf16"), (40, 1030, 4112, 64, "f32"),
    (2048, 1000, 688, 128, "f32"), (9, 700, 2048, 128, "f32"),
])
def test_nothing_behind_the_workspace_is_written(dev, M, N, K, r, y_type):
    import torch
    say("fp8_lora_linear in its room", M, N, K, r, y_type)
    c = Linear(M + K, M, N, K, r, dev)
    ws, behind = guarded(H.hydra_fp8_lora_linear_workspace_bytes(M, N, K, r), dev)
    y = c.forward(y_type, workspace=ws)
    torch.cuda.synchronize()
    assert (behind == BYTE).all()
    at = some(M)
    A, B = c.ab()
    x = f64(c.x)[at]
    ref = fp8_linear_ref(x, c.W, A, B, S)
    tol = linear_bounds(dequantize_ref(*quantize_ref(x, 1), 1), c.W, A, B, S, y_type, x)
    for g, e, t, name in zip(y, ref, tol, ("y_off", "y_on")):
        assert not torch.isnan(g).any()
        near(f64(g)[at], e, rounded(t, e, y_type), name)


@pytest.mark.parametrize("M,N,K,r,dx_type,p", [
    (1280, 11008, 4096, 16, "f32", 0.0), (2100, 8192, 2048, 16, "f32", 0.1), (3585, 12288, 1040, 16, "bf16", 0.0),
    (250, 8192, 2048, 128, "f32", 0.0), (40, 4112, 1040, 64, "bf16", 0.1), (700, 688, 1008, 100, "f32", 0.0),
])
def test_no_stage_of_the_backward_overwrites_another(dev, M, N, K, r, dx_type, p):
    import torch
    say("fp8_lora_linear_backward in its room", M, N, K, r, dx_type, p)
    c = Linear(M + N, M, N, K, r, dev)
    ws, behind = guarded(H.hydra_fp8_lora_linear_backward_workspace_bytes(M, N, K, r), dev)
    dx, dA, dB = empty((M, K), dx_type, dev), empty((r, K), "f32", dev), empty((N, r), "f32", dev)
    rng = rng_of(11, 3, dev)
    H.hydra_fp8_lora_linear_backward(c.xa, c.qt, c.st, c.A, c.B, S, c.dy, dx, dA, dB, p=p, rng=rng, workspace=ws)
    torch.cuda.synchronize()
    assert (behind == BYTE).all()
    mask = torch.empty((M, K), device=dev)  # (pinned element by element in the tests of dropout)
    H.hydra_dropout(torch.ones((M, K), device=dev), mask, p, rng)
    at = some(M)
    A, B = c.ab()
    xa, dy, factor = f64(c.xa), f64(c.dy), f64(mask)[at]
    ref = fp8_linear_backward_ref(xa[at], c.W, A, B, S, dy[at], factor)[0]
    tol = backward_bounds(xa[at], c.W, A, B, S, dy[at], dx_type, factor)[0]
    near(f64(dx)[at], ref, rounded(tol, ref, dx_type), "dx")
    assert not torch.isnan(dx).any()
    # dA and dB take every row; the base product has no part in them
    u, t = S * (np.abs(dy) @ np.abs(B)), S * (np.abs(xa) @ np.abs(A).T)
    near(f64(dA), S * (dy @ B).T @ xa, ((N + 2.5 + 3 * M + 2) * U) * (u.T @ np.abs(xa)) + 1e-40, "dA")
    near(f64(dB), S * dy.T @ (xa @ A.T), ((K + 2.5 + 3 * M + 2) * U) * (np.abs(dy).T @ t) + 1e-40, "dB")
