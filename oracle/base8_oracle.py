"""Plain float64 CPU oracle for the operators around a frozen base in 8 bits: quantization, the linear and its gradients,
dropout from a counter-based generator, and the verification of drafted tokens.

TEST INFRASTRUCTURE ONLY.  Nothing on the product path may import, call or execute this module.  It shares no code
with the HIP library and imports nothing from it.  Inputs are numpy arrays, taken as float64 values.

* e4m3 (OCP): 1 sign, 4 exponent and 3 fraction bits, bias 7; 0x7F and 0xFF are NaN, nothing is infinite, the largest is
  448.  A block's scale is 2^e, e the least integer >= -127 that brings its largest finite magnitude to 448 or less; a
  value becomes the nearest e4m3 value of x 2^-e (ties to the even code), NaN and infinities become NaN.
* Philox4x32-10: the published generator (ten rounds of two 32 x 32 -> 64 bit products).  Element i takes half i % 2 (the
  lower first) of word (i % 8) / 2 of block i / 8, whose counter is (i / 8, offset), key the seed.
* Drafted tokens: accepted while u q < p; the next token from max(p - q, 0), or from p after the last, by the first
  index whose running sum exceeds u of the total.

Pins: see ``tests/test_oracle_base8_pins.py`` (code tables, published test vectors, exact distributions, differences,
planted mistakes).
"""
from __future__ import annotations

import numpy as np

__all__ = ["e4m3_values", "quantize_ref", "dequantize_ref", "fp8_linear_ref", "fp8_linear_backward_ref", "philox_ref",
           "dropout_bits_ref", "dropout_factor_ref", "verify_ref"]

BLOCK = 128


def e4m3_values():
    """The value of each of the 256 codes."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        a = np.ldexp(1 + m / 8, e - 7) if e else np.ldexp(m / 8, -6)
        v[c] = np.nan if (c & 127) == 127 else -a if c >> 7 else a
    return v


VALUES = e4m3_values()


def _round(v):
    """The nearest e4m3 value to each v of magnitude 448 at most, by the distance to the two neighbours."""
    mags = VALUES[:127]
    a = np.abs(v)
    hi = np.clip(np.searchsorted(mags, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = mags[hi] - a, a - mags[lo]
    code = np.where(up < down, hi, np.where(up > down, lo, np.where(hi % 2 == 0, hi, lo)))
    return np.copysign(mags[code], v)


def quantize_ref(x, rows: int):
    """(values q [M, K], whole e [ceil(M / rows), ceil(K / 128)])."""
    x = np.asarray(x, np.float64)
    M, K = x.shape
    q = np.empty((M, K))
    e = np.empty((-(-M // rows), -(-K // BLOCK)), np.int64)
    for i in range(e.shape[0]):
        for j in range(e.shape[1]):
            at = (slice(i * rows, (i + 1) * rows), slice(j * BLOCK, (j + 1) * BLOCK))
            b = x[at]
            fine = np.isfinite(b)
            a = np.abs(b[fine]).max() if fine.any() else 0.0
            n = -127
            if a > 0:
                n = max(n, int(np.floor(np.log2(a / 448))) - 1)
                while a > 448 * 2.0 ** n:
                    n += 1
            e[i, j] = n
            q[at] = np.where(fine, _round(np.where(fine, b, 0.0) * 2.0 ** -n), np.nan)
    return q, e


def dequantize_ref(q, e, rows: int):
    q = np.asarray(q, np.float64)
    M, K = q.shape
    return q * np.exp2(np.repeat(np.repeat(np.asarray(e, np.float64), rows, 0)[:M], BLOCK, 1)[:, :K])


def fp8_linear_ref(x, Wh, A=None, B=None, s: float = 0.0, xa=None):
    """(y_off, y_on) for the values Wh of the quantized weight."""
    x = np.asarray(x, np.float64)
    y = dequantize_ref(*quantize_ref(x, 1), 1) @ np.asarray(Wh, np.float64).T
    if A is None or len(A) == 0:
        return y, y.copy()
    xa = x if xa is None else np.asarray(xa, np.float64)
    return y, y + s * ((xa @ np.asarray(A, np.float64).T) @ np.asarray(B, np.float64).T)


def fp8_linear_backward_ref(xa, Wh, A, B, s: float, dy, factor=None, quantize: bool = True):
    """(dx, dA, dB); factor: what dropout multiplies the adapter's input by.  quantize False: the gradients of the
    function of the values (dy as it is)."""
    xa, Wh, A, B, dy = (np.asarray(a, np.float64) for a in (xa, Wh, A, B, dy))
    u = s * (dy @ B)
    through = u @ A
    if factor is not None:
        through = np.where(factor != 0, through * factor, 0.0)
    base = dequantize_ref(*quantize_ref(dy, 1), 1) if quantize else dy
    return base @ Wh + through, u.T @ xa, s * (dy.T @ (xa @ A.T))


def philox_ref(counter, key):
    """The four words of one block."""
    c, k = [int(v) for v in counter], [int(v) for v in key]
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_bits_ref(seed: int, offset: int, index):
    """The sixteen bits of each element."""
    seed, offset = seed % (1 << 64), offset % (1 << 64)
    bits = []
    for i in np.asarray(index).ravel().tolist():
        g = i // 8
        w = philox_ref((g & 0xFFFFFFFF, g >> 32, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32))
        bits.append((w[i % 8 // 2] >> (16 * (i % 2))) & 0xFFFF)
    return np.array(bits, np.int64).reshape(np.shape(index))


def dropout_factor_ref(seed: int, offset: int, p: float, shape):
    n = int(np.prod(shape))
    d = round(p * 65536)
    keep = dropout_bits_ref(seed, offset, np.arange(n)) >= d
    return (keep * (65536 / (65536 - d) if d < 65536 else 0.0)).reshape(shape)


def verify_ref(target, draft, drafts, lens, u, T: float = 1.0):
    """(accepted, tokens, lp, odd) for target [n, k + 1, V], draft [n, k, V] or None; odd: whether something was out of
    order (see the library's err_flag)."""
    target, u = np.asarray(target, np.float64), np.asarray(u, np.float64)
    n, k1, V = target.shape
    k = k1 - 1

    def softmax(z):
        """(probabilities, their logarithms), or None for a row without a distribution."""
        if np.isnan(z).any() or (z == np.inf).any() or (z == -np.inf).all():
            return None
        with np.errstate(over="ignore", under="ignore"):
            c = (z - z.max()) / T
            w = np.exp(c)
            return w / w.sum(), c - np.log(w.sum())

    acc, tok, lps, odd = np.zeros(n, np.int64), np.full((n, k1), -1, np.int64), np.zeros((n, k1)), False
    for b in range(n):
        length = k if lens is None else int(lens[b])
        odd |= not 0 <= length <= k
        length = min(max(length, 0), k)
        for j in range(length + 1):
            s = softmax(target[b, j])
            if s is None:
                lps[b, j], odd = np.nan, True
                break
            p, lp = s
            left = p
            if j < length:
                t = int(drafts[b][j])
                q = None
                if 0 <= t < V:
                    if draft is None:
                        q = np.zeros(V)
                        q[t] = 1.0
                    else:
                        sd = softmax(np.asarray(draft, np.float64)[b, j])
                        q = None if sd is None else sd[0]
                if q is None:
                    odd = True
                else:
                    if u[b, j] * q[t] < p[t]:
                        tok[b, j], lps[b, j] = t, lp[t]
                        acc[b] += 1
                        continue
                    left = np.maximum(p - q, 0.0)
                    if not left.sum() > 0:
                        left = p
            sums = np.cumsum(left)
            past = np.nonzero((sums > u[b, k] * sums[-1]) & (left > 0))[0]
            v = past[0] if past.size else np.nonzero(left > 0)[0][-1]
            tok[b, j], lps[b, j] = v, lp[v]
            break
    return acc, tok, lps, odd
