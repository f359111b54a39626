"""Pins of the update-step oracle (layer norm, token log-probabilities, gradient norm) against things other than itself:
differences of the forwards, closed forms, float64 autograd on the CPU, and planted mistakes."""
import math

import numpy as np
import pytest
import torch

from oracle import update_oracle as U


def _ln_case(seed=0, M=3, K=5):
    r = np.random.default_rng(seed)
    return r.normal(0.3, 1.5, (M, K)), r.normal(1, 0.2, K), r.normal(0, 0.3, K), r.normal(0, 1, (M, K))


def _backward_error(f):
    """Largest difference of f's gradients from central differences of sum(dy * y)."""
    x, w, b, dy = _ln_case()
    _, mean, rstd = U.layer_norm_ref(x, w, b, 1e-3)
    got = f(dy, x, w, mean, rstd)
    h, worst = 1e-5, 0.0
    for a, g in zip((x, w, b), got):
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + h
            up = (dy * U.layer_norm_ref(x, w, b, 1e-3)[0]).sum()
            a[i] = keep - h
            dn = (dy * U.layer_norm_ref(x, w, b, 1e-3)[0]).sum()
            a[i] = keep
            worst = max(worst, abs((up - dn) / (2 * h) - g[i]))
    return worst


def test_layer_norm_closed_forms():
    x = np.array([[1.0, 3.0], [-2.0, -2.0]])
    y, mean, rstd = U.layer_norm_ref(x, eps=1e-9)
    assert np.allclose(mean, [2, -2]) and np.allclose(y[0], [-1, 1], atol=1e-8) and np.all(y[1] == 0)
    assert math.isclose(rstd[1], 1e-9 ** -0.5)
    y, _, _ = U.layer_norm_ref(x * 7 + 11, eps=1e-12)  # shift and scale leave it alone
    assert np.allclose(y[0], [-1, 1])
    y, _, _ = U.layer_norm_ref([[5.0]], [3.0], [0.25])
    assert y[0, 0] == 0.25


def test_layer_norm_matches_torch():
    x, w, b, dy = (torch.tensor(a, requires_grad=True) for a in _ln_case(1, 4, 33))
    y = torch.nn.functional.layer_norm(x, (33,), w, b, 1e-5)
    y.backward(dy.detach())
    e, mean, rstd = U.layer_norm_ref(x.detach(), w.detach(), b.detach())
    assert np.allclose(e, y.detach().numpy(), atol=1e-12)
    for g, t in zip(U.layer_norm_backward_ref(dy.detach(), x.detach(), w.detach(), mean, rstd), (x, w, b)):
        assert np.allclose(g, t.grad.numpy(), atol=1e-12)


def test_layer_norm_gradient_by_differences():
    assert _backward_error(U.layer_norm_backward_ref) < 1e-8


def test_planted_mistakes_in_the_layer_norm_gradient_are_found():
    def no_mean(dy, x, w, mean, rstd):
        dx, dw, db = U.layer_norm_backward_ref(dy, x, w, mean, rstd)
        return dx + rstd[:, None] * (dy * w).mean(1, keepdims=True), dw, db

    def no_weight(dy, x, w, mean, rstd):
        return (U.layer_norm_backward_ref(dy, x, None, mean, rstd)[0], *U.layer_norm_backward_ref(dy, x, w, mean, rstd)[1:])

    def weighted_dw(dy, x, w, mean, rstd):
        dx, dw, db = U.layer_norm_backward_ref(dy, x, w, mean, rstd)
        return dx, dw * w, db

    for f in (no_mean, no_weight, weighted_dw):
        assert _backward_error(f) > 1e-3, f.__name__


def test_token_logprobs_closed_forms():
    o = U.token_logprobs_ref(np.zeros((1, 8)), [3], 3)
    assert math.isclose(o["lp"][0], -math.log(8)) and math.isclose(o["entropy"][0], math.log(8))
    assert list(o["ids"][0]) == [0, 1, 2]
    d = 1.75
    o = U.token_logprobs_ref([[0.0, -d]], [1], 2)
    p = 1 / (1 + math.exp(-d))
    assert math.isclose(o["lp"][0], -math.log1p(math.exp(d)))
    assert math.isclose(o["entropy"][0], -p * math.log(p) - (1 - p) * math.log(1 - p))
    o = U.token_logprobs_ref([[2.0, -np.inf, 2.0]], [0], 3)
    assert math.isclose(o["entropy"][0], math.log(2)) and list(o["ids"][0]) == [0, 2, 1] and o["top_lp"][0][2] == -np.inf
    o = U.token_logprobs_ref([[-np.inf, -np.inf]], [0], 1)
    assert o["lse"][0] == -np.inf and np.isnan(o["lp"][0]) and np.isnan(o["entropy"][0]) and o["ids"][0][0] == 0
    o = U.token_logprobs_ref([[1.0, np.nan, np.inf, np.nan]], [0], 3)
    assert list(o["ids"][0]) == [1, 3, 2] and np.isnan(o["lse"][0])
    low = float(np.finfo(np.float32).min)
    o = U.token_logprobs_ref([[low, low, low, low]], [2], 1)
    assert math.isclose(o["entropy"][0], math.log(4)) and math.isclose(o["lp"][0], -math.log(4))
    assert math.isnan(U.token_logprobs_ref([[0.0]], [1])["lp"][0])


def test_token_logprobs_match_torch():
    r = np.random.default_rng(4)
    z = torch.tensor(r.normal(0, 2, (5, 40)), requires_grad=True)
    tok = torch.tensor([0, 39, 7, 7, 20])
    d_lp, d_h = torch.tensor(r.normal(0, 1, 5)), torch.tensor(r.normal(0, 1, 5))
    lp = torch.log_softmax(z, 1)
    h = -(lp.exp() * lp).sum(1)
    (lp.gather(1, tok[:, None])[:, 0] * d_lp + h * d_h).sum().backward()
    o = U.token_logprobs_ref(z.detach(), tok.numpy(), 4)
    assert np.allclose(o["lp"], lp.gather(1, tok[:, None])[:, 0].detach()) and np.allclose(o["entropy"], h.detach())
    assert np.array_equal(o["ids"], torch.topk(z, 4).indices.numpy())
    g = U.token_logprobs_backward_ref(z.detach(), tok.numpy(), o["lse"], d_lp.numpy(), o["entropy"], d_h.numpy())
    assert np.allclose(g, z.grad.numpy(), atol=1e-14)
    assert np.allclose(g.sum(1), 0, atol=1e-14)  # logits shifted by one number change nothing


def _lp_backward_error(f):
    r = np.random.default_rng(5)
    z, tok = r.normal(0, 1.5, (2, 6)), [4, 0]
    d_lp, d_h = r.normal(0, 1, 2), r.normal(0, 1, 2)

    def loss():
        o = U.token_logprobs_ref(z, tok)
        return (o["lp"] * d_lp + o["entropy"] * d_h).sum()

    o = U.token_logprobs_ref(z, tok)
    g, h, worst = f(z, tok, o["lse"], d_lp, o["entropy"], d_h), 1e-5, 0.0
    for i in np.ndindex(z.shape):
        keep = z[i]
        z[i] = keep + h
        up = loss()
        z[i] = keep - h
        dn = loss()
        z[i] = keep
        worst = max(worst, abs((up - dn) / (2 * h) - g[i]))
    return worst


def test_token_logprobs_gradient_by_differences():
    assert _lp_backward_error(U.token_logprobs_backward_ref) < 1e-9


def test_planted_mistakes_in_the_logprob_gradient_are_found():
    full = U.token_logprobs_backward_ref

    def no_token(z, tok, lse, a, h, e):
        g = full(z, tok, lse, a, h, e)
        for m, t in enumerate(tok):
            g[m, t] -= a[m]
        return g

    def sign(z, tok, lse, a, h, e):
        return full(z, tok, lse, a, h, -e)

    def no_entropy(z, tok, lse, a, h, e):
        return full(z, tok, lse, a, 0 * h, e)

    for f in (no_token, sign, no_entropy):
        assert _lp_backward_error(f) > 1e-3, f.__name__


def test_rows_without_an_upstream_gradient():
    z = np.array([[np.nan, 1.0], [0.0, 0.0]])
    g = U.token_logprobs_backward_ref(z, [9, 9], [np.nan, np.log(2)], [0.0, 1.0])
    assert np.all(g[0] == 0) and np.isnan(g[1]).all()


def test_grad_norm_and_clip():
    assert U.grad_norm_ref([[3.0], [[4.0, 0.0]]]) == 5.0
    n, out = U.grad_clip_ref([[3.0], [[4.0, 0.0]]], 1.0)
    assert n == 5.0 and np.allclose(out[0], [0.6]) and np.allclose(out[1], [[0.8, 0.0]])
    assert math.isclose(U.grad_norm_ref(out), 1.0)
    _, out = U.grad_clip_ref([[3.0], [[4.0, 0.0]]], 5.0)  # at the limit nothing changes
    assert np.array_equal(out[0], [3.0])
    n, out = U.grad_clip_ref([[np.inf, 1.0]], 1.0)
    assert n == np.inf and np.array_equal(out[0], [np.inf, 1.0])
    n, out = U.grad_clip_ref([[0.0, 0.0]], 0.0)
    assert n == 0 and np.array_equal(out[0], [0, 0])
