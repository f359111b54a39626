"""Helpers of the GPU tests of layer norm, token log-probabilities and gradient clipping: tensors of either type at any
alignment, and the error bounds, derived from the arithmetic.

U is half a step of fp32.  A sum of n terms in any order is off by at most (n - 1) U times the sum of their magnitudes;
the kernels add n terms as chains of at most n / 64 in each of 64 or more lanes and a tree over the lanes, so that
depth(n) = n / 64 + 16 holds for them.  Rounding a result to bf16 adds 2^-8 of its value.
"""
import numpy as np

U = 2.0 ** -24
TYPES = ("bf16", "f32")


def depth(n):
    return n / 64 + 16


def dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def out_step(name):
    return 2.0 ** -8 if name == "bf16" else U


def put(a, name, dev, shift=0, stride=0):
    """`a` as a device tensor of this type, `shift` elements past a 256-byte boundary, its rows `stride` elements apart
    (0: contiguous; the gaps hold NaN)."""
    import torch
    a = torch.as_tensor(np.asarray(a, np.float32))
    ld = stride or (a.shape[-1] if a.dim() > 1 else 1)
    n = a.numel() if a.dim() < 2 else (a.shape[0] - 1) * ld + a.shape[1]
    flat = torch.full((shift + n + 8,), float("nan"), dtype=dtype(name), device=dev)
    t = flat[shift:shift + n]
    t = t.view(a.shape) if a.dim() < 2 or ld == a.shape[1] else t.as_strided(a.shape, (ld, 1), shift)
    t.copy_(a)
    return t


def empty(shape, name, dev, shift=0, stride=0):
    return put(np.full(shape, np.nan), name, dev, shift, stride)


def f64(t):
    return t.detach().to("cpu").double().numpy()


def near(got, ref, tol, what):
    """|got - ref| <= tol everywhere, NaN where and only where ref has it, infinities equal."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    tol = np.broadcast_to(np.asarray(tol, np.float64), ref.shape)
    assert got.shape == ref.shape, f"{what}: {got.shape} for {ref.shape}"
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN in {np.isnan(got).sum()} places, not {np.isnan(ref).sum()}"
    # (neither type holds a number of 2^128 or more: it rounds to an infinity)
    ref = np.where(np.abs(ref) >= 2.0 ** 128, np.copysign(np.inf, ref), ref)
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]), f"{what}: infinities"
    ok = ~inf & ~np.isnan(ref)
    off = np.abs(got[ok] - ref[ok]) / np.maximum(tol[ok], 1e-300)
    assert off.size == 0 or off.max() <= 1, f"{what}: {off.max():.2f} times the bound at {int(off.argmax())}"


def norm_bounds(x, w, b, y_type, eps=1e-5):
    """Bounds of y, mean, rstd: the mean's sum, the centred values (one rounding and the mean's error), their squares'
    sum, the root, two products and an addition, the result's type."""
    x = np.asarray(x, np.float64)
    K = x.shape[1]
    mean = x.mean(1, keepdims=True)
    c = x - mean
    e_mean = U * ((depth(K) + 2) * np.abs(x).mean(1, keepdims=True) + np.abs(mean))
    var = (c * c).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    # the variance of values off by e_mean and a rounding, relative to var + eps; half of it in rstd
    e_var = (2 * (e_mean + U * np.abs(c).max(1, keepdims=True)) * np.abs(c).mean(1, keepdims=True) + e_mean ** 2
             + U * (depth(K) + 4) * var + U * var)
    r_rstd = 0.5 * e_var / (var + eps) + 4 * U
    w = np.ones(K) if w is None else np.asarray(w, np.float64)
    b = np.zeros(K) if b is None else np.asarray(b, np.float64)
    y = c * rstd * w + b
    e_y = np.abs(w) * rstd * (e_mean + np.abs(c) * (r_rstd + 4 * U)) + U * (np.abs(y) + np.abs(b))
    return e_y + (out_step(y_type) * (np.abs(y) + e_y) + 1e-40 if y_type == "bf16" else 0), e_mean[:, 0], (rstd * r_rstd)[:, 0]


def norm_back_bounds(dy, x, w, mean, rstd, dx_type):
    """Bounds of dx, dw, db for given mean and rstd."""
    dy, x, mean, rstd = (np.asarray(a, np.float64) for a in (dy, x, mean, rstd))
    mean, rstd = mean[:, None], rstd[:, None]
    M, K = x.shape
    xh = (x - mean) * rstd
    g = dy * (1 if w is None else np.asarray(w, np.float64))
    r_xh = 3 * U  # of xh's own size
    c1, c2 = g.mean(1, keepdims=True), (g * xh).mean(1, keepdims=True)
    e1 = U * (depth(K) + 3) * np.abs(g).mean(1, keepdims=True)
    e2 = (U * (depth(K) + 4) + r_xh) * np.abs(g * xh).mean(1, keepdims=True)
    dx = rstd * (g - c1 - xh * c2)
    e_dx = rstd * (e1 + np.abs(xh) * e2 + (r_xh + 4 * U) * (np.abs(g) + np.abs(c1) + np.abs(xh * c2)))
    if dx_type == "bf16":
        e_dx = e_dx + out_step(dx_type) * (np.abs(dx) + e_dx) + 1e-40
    e_dw = (U * (M + 4) + r_xh) * np.abs(dy * xh).sum(0)
    return e_dx, e_dw + 1e-40, U * (M + 4) * np.abs(dy).sum(0) + 1e-40


def logp_bounds(z, ref):
    """Bounds of lse, entropy and, as a function of the logits asked for, of log-probabilities.  An exponential is off by
    (|d| + 3) U of itself for d = z - max (the difference's and the product's rounding); mean_d is the mean of |d| under
    the distribution."""
    z = np.asarray(z, np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        most = z.max(1)
        d = np.where(np.isneginf(z), 0.0, most[:, None] - z)
        p = np.exp(z - ref["lse"][:, None])
        p = np.where(np.isfinite(p), p, 0.0)
        mean_d = (p * np.minimum(d, 1e4)).sum(1)
    n = depth(z.shape[1])
    r_s = U * (n + 3 * mean_d + 8)                       # of the sum
    with np.errstate(invalid="ignore"):
        e_lse = r_s + U * (np.abs(ref["lse"]) + np.abs(ref["lse"] - most) + 2)
    e_h = r_s * (2 + 2 * mean_d) + U * (n + 8) * mean_d + 3 * U * (np.abs(ref["entropy"]) + 1)

    def e_lp(asked):
        return e_lse + U * (np.abs(asked) + np.abs(ref["lse"]) + np.abs(asked - ref["lse"]))

    return e_lse, e_h, e_lp


def logp_back_bounds(z, lse, d_lp, entropy, d_entropy, ref, d_type):
    """Bounds of the gradient for given lse and entropy."""
    z, lse = np.asarray(z, np.float64), np.asarray(lse, np.float64)[:, None]
    a = np.zeros_like(lse) if d_lp is None else np.abs(np.asarray(d_lp, np.float64))[:, None]
    e = np.zeros_like(lse) if d_entropy is None else np.abs(np.asarray(d_entropy, np.float64))[:, None]
    h = np.zeros_like(lse) if entropy is None else np.asarray(entropy, np.float64)[:, None]
    with np.errstate(invalid="ignore", over="ignore"):
        lp = np.where(np.isneginf(z), -1e4, z - lse)
        p = np.exp(lp)
        r_p = U * (3 * np.abs(lp) + 4)
        tol = p * (a * (r_p + 3 * U) + e * (np.abs(lp + h) * (r_p + 4 * U) + U * (2 * np.abs(lp) + np.abs(h))))
        tol = tol + 2 * U * (a + np.abs(ref))
        if d_type == "bf16":
            tol = tol + out_step(d_type) * (np.abs(ref) + tol)
    return np.where(np.isfinite(tol), tol, 0.0) + 1e-37  # (below it fp32 and bf16 have no whole mantissa)
