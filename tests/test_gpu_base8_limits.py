"""The 8-bit base beyond 2^32 elements (weights, activations, logits' strides), at the largest K, and scale bytes that a
quantization does not make."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import (dequantize_ref, dropout_bits_ref, fp8_linear_backward_ref, fp8_linear_ref, quantize_ref, verify_ref)
from base8_helpers import backward_bounds, bytes_of, linear_bounds, quantized, rng_of, rounded, values_of
from gpu_helpers import say
from update_helpers import U, dtype, empty, f64, near, put

pytestmark = pytest.mark.gpu

S = 1.25
LAST = 40


@pytest.fixture(autouse=True)
def leave_no_memory():
    import torch
    yield
    torch.cuda.empty_cache()


def few_codes(shape, dev, seed):
    """e4m3 bytes below 0x70 (up to 160), and their float64 values on demand."""
    import torch
    g = torch.Generator(dev).manual_seed(seed)
    return torch.randint(0, 0x70, shape, generator=g, device=dev, dtype=torch.uint8)


@pytest.mark.parametrize("M", [3, 9, 40])
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
def test_a_weight_of_more_than_2_32_elements(dev, M, y_type):
    import torch
    say("weight beyond 2^32", M, y_type)
    N, K, r = (1 << 20) + 8292, 4112, 8
    rng = np.random.default_rng(M)
    Wq = few_codes((N, K), dev, 1)
    ws = torch.randint(118, 124, (-(-N // 128), -(-K // 128)), device=dev, dtype=torch.uint8)
    x, A = put(rng.normal(0, 1, (M, K)), "bf16", dev), put(rng.normal(0, K ** -0.5, (r, K)), "bf16", dev)
    B = torch.randn((N, r), device=dev).bfloat16()
    y = [torch.full((M, N), float("nan"), dtype=dtype(y_type), device=dev) for _ in range(2)]
    H.hydra_fp8_lora_linear(x, Wq, ws, A, B, S, *y)
    torch.cuda.synchronize()
    rows = np.r_[0:8, N - LAST:N]
    at = torch.as_tensor(rows).to(dev)
    e = ws.cpu().numpy().astype(np.int64)[rows // 128] - 127
    W = values_of(Wq[at]) * 2.0 ** np.repeat(e, 128, 1)[:, :K]
    ref = fp8_linear_ref(f64(x), W, f64(A), f64(B[at]), S)
    tol = linear_bounds(dequantize_ref(*quantize_ref(f64(x), 1), 1), W, f64(A), f64(B[at]), S, y_type, f64(x))
    for g, v, t, name in zip(y, ref, tol, ("y_off", "y_on")):
        near(f64(g[:, at]), v, rounded(t, v, y_type), name)


@pytest.mark.parametrize("y_type", ["f32", "bf16"])
def test_rows_of_more_than_2_32_elements(dev, y_type):
    """Quantization, linear, and the backward's dx under its mask: the last rows."""
    import torch
    say("rows beyond 2^32", y_type)
    M, K, N, r, p = 1 << 20, 4112, 48, 8, 0.25
    rng = np.random.default_rng(2)
    g = torch.Generator(dev).manual_seed(3)
    x = torch.empty((M, K), dtype=torch.bfloat16, device=dev).normal_(generator=g)
    (q, s, qt, st), W = quantized(f64(put(rng.normal(0, 0.02, (N, K)), "bf16", dev)), dev)
    A, B = put(rng.normal(0, K ** -0.5, (r, K)), "bf16", dev), put(rng.normal(0, 0.3, (N, r)), "bf16", dev)
    last = f64(x[-LAST:])
    xh = quantize_ref(last, 1)
    xq = torch.empty((M, K), dtype=torch.uint8, device=dev)
    xs = torch.empty((M, -(-K // 128)), dtype=torch.uint8, device=dev)
    H.hydra_fp8_quantize(x, xq, xs)
    assert np.array_equal(values_of(xq[-LAST:]), xh[0]) and np.array_equal(bytes_of(xs[-LAST:]), xh[1] + 127)
    del xq, xs
    y = [torch.full((M, N), float("nan"), dtype=dtype(y_type), device=dev) for _ in range(2)]
    H.hydra_fp8_lora_linear(x, q, s, A, B, S, *y)
    ref = fp8_linear_ref(last, W, f64(A), f64(B), S)
    tol = linear_bounds(dequantize_ref(*xh, 1), W, f64(A), f64(B), S, y_type, last)
    for got, v, t, name in zip(y, ref, tol, ("y_off", "y_on")):
        near(f64(got[-LAST:]), v, rounded(t, v, y_type), name)
    del y
    dy = torch.empty((M, N), dtype=torch.bfloat16, device=dev).normal_(generator=g)
    dx = torch.full((M, K), float("nan"), dtype=dtype(y_type), device=dev)
    H.hydra_fp8_lora_linear_backward(None, qt, st, A, B, S, dy, dx, p=p, rng=rng_of(5, 6, dev))
    torch.cuda.synchronize()
    n = 2
    d = f64(dy[-LAST:])
    factor = np.ones((LAST, K))
    index = np.arange((M - n) * K, M * K).reshape(n, K)
    factor[-n:] = (dropout_bits_ref(5, 6, index) >= 65536 * p) / (1 - p)
    ref = fp8_linear_backward_ref(last, W, f64(A), f64(B), S, d, factor)[0]
    tol = backward_bounds(last, W, f64(A), f64(B), S, d, y_type, factor)[0]
    near(f64(dx[-n:]), ref[-n:], rounded(tol, ref, y_type)[-n:], "dx")


@pytest.mark.parametrize("M", [2, 17])
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
def test_the_largest_k(dev, M, y_type):
    say("largest K", M, y_type)
    K, N, r = 1 << 21, 5, 2
    rng = np.random.default_rng(M)
    x, A = put(rng.normal(0, 1, (M, K)), "bf16", dev), put(rng.normal(0, K ** -0.5, (r, K)), "bf16", dev)
    (q, s, _, _), W = quantized(f64(put(rng.normal(0, 0.02, (N, K)), "bf16", dev)), dev)
    B = put(rng.normal(0, 0.3, (N, r)), "bf16", dev)
    y = [empty((M, N), y_type, dev) for _ in range(2)]
    H.hydra_fp8_lora_linear(x, q, s, A, B, S, *y)
    ref = fp8_linear_ref(f64(x), W, f64(A), f64(B), S)
    tol = linear_bounds(dequantize_ref(*quantize_ref(f64(x), 1), 1), W, f64(A), f64(B), S, y_type, f64(x))
    for g, v, t, name in zip(y, ref, tol, ("y_off", "y_on")):
        near(f64(g), v, rounded(t, v, y_type), name)


def test_logits_more_than_2_32_elements_apart(dev):
    import torch
    say("logits far apart")
    n, k, V, ld = 2, 2, 5000, (1 << 30) + 4
    r = np.random.default_rng(4)
    z, zd = r.normal(0, 2, (n * (k + 1), V)), r.normal(0, 2, (n * k, V))

    def apart(a):
        flat = torch.empty((len(a) - 1) * ld + V, dtype=torch.bfloat16, device=dev)
        t = flat.as_strided(a.shape, (ld, 1))
        t.copy_(torch.as_tensor(a))
        return t

    z, zd = apart(z), apart(zd)
    drafts = r.integers(0, V, (n, k)).astype(np.int32)
    u = r.uniform(0, 1, (n, k + 1)).astype(np.float32)
    u[1, :k] = 0
    acc, tok, lp = (torch.zeros(s, dtype=t, device=dev) for s, t in (((n,), torch.int32), ((n, k + 1), torch.int32),
                                                                     ((n, k + 1), torch.float32)))
    H.hydra_verify_drafts(z, zd, torch.as_tensor(drafts).to(dev), torch.as_tensor(u).to(dev), acc, tok, lp)
    torch.cuda.synchronize()
    ref = verify_ref(f64(z).reshape(n, k + 1, V), f64(zd).reshape(n, k, V), drafts, None, u)
    assert np.array_equal(acc.cpu().numpy(), ref[0]) and np.array_equal(tok.cpu().numpy(), ref[1]) and ref[0][1] == k
    near(f64(lp), ref[2], U * np.abs(ref[2]) + 1e-9, "lp")


@pytest.mark.parametrize("M", [3, 40])
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
def test_a_scale_byte_of_255_is_nan(dev, M, y_type):
    import torch
    say("scale 255", M, y_type)
    N, K = 150, 400
    rng = np.random.default_rng(5)
    (q, s, _, _), W = quantized(f64(put(rng.normal(0, 1, (N, K)), "bf16", dev)), dev)
    x = put(rng.normal(0, 1, (M, K)), "bf16", dev)
    xq, xs = torch.empty((M, K), dtype=torch.uint8, device=dev), torch.empty((M, 4), dtype=torch.uint8, device=dev)
    H.hydra_fp8_quantize(x, xq, xs)
    s[1, 2] = 255
    xs[1, 3] = 255
    y = empty((M, N), y_type, dev)
    H.hydra_fp8_lora_linear(None, q, s, None, None, 0.0, y, xq=xq, x_scale=xs)
    bad = np.zeros((M, N), bool)
    bad[1], bad[:, 128:] = True, True
    assert np.array_equal(np.isnan(f64(y)), bad)
