"""Plain float64 CPU oracle for the operators of an update step around the PPO losses and the linear's backward.

TEST INFRASTRUCTURE ONLY.  Nothing on the product path may import, call or execute this module.  It shares no code
with the HIP library and imports nothing from it.  Inputs are numpy arrays, taken as float64 values.

* Layer norm over the last axis and its gradients: the variance is that of the K values (divided by K), eps is added to
  it under the root.  The gradients are those of ``sum(dy * y)`` with mean and rstd as functions of x; the functions
  take the forward's mean and rstd as given numbers.
* Log-probabilities of given tokens, the distribution's entropy and the ``top`` most likely entries (greatest first,
  the lowest index first among equals, NaN before every number), and the gradient of ``sum(d_lp * lp + d_entropy * H)``
  with respect to the logits, with the forward's lse and entropy as given numbers.  Masked-out entries (-inf) have
  probability 0.  A row without an upstream gradient has gradient 0.
* The norm over many tensors, and the tensors scaled to a norm of at most ``max_norm``; nothing is scaled where the norm
  is not finite.

Pins: see ``tests/test_oracle_update_pins.py`` (differences of the forward, closed forms, autograd in float64 and planted
mistakes).
"""
from __future__ import annotations

import numpy as np

__all__ = ["layer_norm_ref", "layer_norm_backward_ref", "token_logprobs_ref", "token_logprobs_backward_ref",
           "grad_norm_ref", "grad_clip_ref"]


def _f64(a):
    return np.asarray(a, np.float64)


def layer_norm_ref(x, w=None, b=None, eps: float = 1e-5):
    """(y, mean, rstd)."""
    x = _f64(x)
    K = x.shape[1]
    mean = x.sum(1) / K
    c = x - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).sum(1) / K + eps)
    y = c * rstd[:, None]
    if w is not None:
        y = y * _f64(w)
    if b is not None:
        y = y + _f64(b)
    return y, mean, rstd


def layer_norm_backward_ref(dy, x, w, mean, rstd):
    """(dx, dw, db)."""
    dy, x, mean, rstd = _f64(dy), _f64(x), _f64(mean)[:, None], _f64(rstd)[:, None]
    K = x.shape[1]
    xh = (x - mean) * rstd
    g = dy if w is None else dy * _f64(w)
    dx = rstd * (g - g.sum(1, keepdims=True) / K - xh * ((g * xh).sum(1, keepdims=True) / K))
    return dx, (dy * xh).sum(0), dy.sum(0)


def token_logprobs_ref(z, tokens=None, top: int = 0):
    """dict with lp, lse, entropy, ids, top_lp; row by row."""
    z = _f64(z)
    M, V = z.shape
    o = {"lp": np.full(M, np.nan), "lse": np.empty(M), "entropy": np.empty(M), "ids": np.empty((M, top), np.int64),
         "top_lp": np.empty((M, top))}
    for m in range(M):
        row = z[m]
        order = sorted(range(V), key=lambda j: (0 if np.isnan(row[j]) else 1, -row[j] if not np.isnan(row[j]) else 0.0, j))[
            :top] if top else []
        o["ids"][m] = order
        if np.isnan(row).any() or (row == np.inf).any():
            o["lse"][m] = o["entropy"][m] = np.nan
            o["top_lp"][m] = np.nan
            continue
        most = row.max()
        if most == -np.inf:
            o["lse"][m], o["entropy"][m] = -np.inf, np.nan
            o["top_lp"][m] = np.nan
            continue
        live = row[row != -np.inf]
        with np.errstate(over="ignore"):
            lse = most + np.log(np.exp(live - most).sum())
            lp = row - lse
            p = np.exp(live - lse)
        if abs(most) > 1e30:  # lse - most is lost in lse itself: by the differences to the largest
            rest = np.log(np.exp(live - most).sum())
            lp, p = (row - most) - rest, np.exp((live - most) - rest)
        llp = lp[row != -np.inf]
        o["lse"][m] = lse
        o["entropy"][m] = -(p[p > 0] * llp[p > 0]).sum()
        o["top_lp"][m] = lp[order] if top else []
        if tokens is not None and 0 <= tokens[m] < V:
            o["lp"][m] = lp[tokens[m]]
    return o


def token_logprobs_backward_ref(z, tokens, lse, d_lp=None, entropy=None, d_entropy=None):
    """The gradient [M, V]."""
    z = _f64(z)
    M, V = z.shape
    d = np.zeros((M, V))
    for m in range(M):
        a = 0.0 if d_lp is None else float(d_lp[m])
        e = 0.0 if d_entropy is None else float(d_entropy[m])
        if a == 0.0 and e == 0.0:
            continue
        if a != 0.0 and not 0 <= tokens[m] < V:
            d[m] = np.nan
            continue
        with np.errstate(over="ignore", invalid="ignore"):
            lp = z[m] - float(lse[m])
            p = np.exp(lp)
        if a != 0.0:
            d[m] -= a * p
            d[m, tokens[m]] += a
        if e != 0.0:
            some = p != 0
            d[m, some] -= e * p[some] * (lp[some] + float(entropy[m]))
    return d


def grad_norm_ref(grads) -> float:
    return float(np.sqrt(sum((_f64(g).ravel() ** 2).sum() for g in grads)))


def grad_clip_ref(grads, max_norm: float):
    """(norm, scaled tensors)."""
    norm = grad_norm_ref(grads)
    c = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, [_f64(g) * c for g in grads]
