"""Layer norm and its gradients against the float64 oracle: both types of every operand, widths from one value to past
what a workgroup's registers hold, alignments, in place, rows with NaN and infinities, values far from zero."""
import itertools

import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import layer_norm_backward_ref, layer_norm_ref
from gpu_helpers import say
from update_helpers import TYPES, empty, f64, near, norm_back_bounds, norm_bounds, put

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 2), (3, 7), (5, 8), (4, 64), (4, 75), (2, 511), (4, 512), (7, 513), (33, 520), (3, 1000), (2, 2047), (5, 2048),
         (2, 2056), (3, 4096), (2, 4099), (2, 8192), (3, 8200), (2, 11008), (2, 16384), (2, 16392), (3, 16385), (1, 40008)]
NAN = float("nan")


def _inputs(M, K, seed, w_type, with_w=True, with_b=True):
    r = np.random.default_rng(seed)
    x = r.normal(0, 1, (M, K)) * r.uniform(0.3, 3, K) + r.normal(0, 0.5, K)
    return x, r.normal(1, 0.2, K) if with_w else None, r.normal(0, 0.3, K) if with_b else None, r.normal(0, 1, (M, K))


def _forward(dev, x, w, b, x_type, w_type, y_type, shift=0, eps=1e-5):
    M, K = x.shape
    xt = put(x, x_type, dev, shift)
    wt, bt = (None if v is None else put(v, w_type, dev, shift) for v in (w, b))
    y, mean, rstd = empty((M, K), y_type, dev, shift), empty(M, "f32", dev, shift), empty(M, "f32", dev, shift)
    H.hydra_layer_norm(xt, wt, bt, y, mean, rstd, eps=eps)
    v = [None if t is None else f64(t) for t in (xt, wt, bt)]
    return v, y, mean, rstd


def _check_forward(v, y, mean, rstd, y_type, eps=1e-5):
    ref = layer_norm_ref(*v, eps)
    for got, r, tol, what in zip((y, mean, rstd), ref, norm_bounds(*v, y_type, eps), ("y", "mean", "rstd")):
        near(f64(got), r, tol, what)


@pytest.mark.parametrize("x_type,w_type,y_type", list(itertools.product(TYPES, TYPES, TYPES)))
def test_forward(x_type, w_type, y_type, dev):
    for i, (M, K) in enumerate(SIZES):
        shift = (0, 0, 1, 4)[i % 4]
        say("layer norm", M, K, x_type, w_type, y_type, shift)
        x, w, b, _ = _inputs(M, K, 100 + K, w_type, i % 5 != 3, i % 5 != 4)
        _check_forward(*_forward(dev, x, w, b, x_type, w_type, y_type, shift), y_type)


def _backward(dev, dy, x, w, dy_type, x_type, w_type, dx_type, shift=0, want=(True, True, True)):
    M, K = x.shape
    dyt, xt, wt = put(dy, dy_type, dev, shift), put(x, x_type, dev, shift), None if w is None else put(w, w_type, dev, shift)
    _, mean, rstd = layer_norm_ref(f64(xt), None, None)
    mt, rt = put(mean, "f32", dev), put(rstd, "f32", dev)
    dx = empty((M, K), dx_type, dev, shift) if want[0] else None
    dw, db = (empty(K, "f32", dev, shift) if k else None for k in want[1:])
    H.hydra_layer_norm_backward(dyt, xt, wt, mt, rt, dx, dw, db)
    return [f64(dyt), f64(xt), None if wt is None else f64(wt), f64(mt), f64(rt)], (dx, dw, db)


def _check_backward(v, got, dx_type):
    for g, r, tol, what in zip(got, layer_norm_backward_ref(*v), norm_back_bounds(*v, dx_type), ("dx", "dw", "db")):
        if g is not None:
            near(f64(g), r, tol, what)


@pytest.mark.parametrize("dy_type,x_type,dx_type", list(itertools.product(TYPES, TYPES, TYPES)))
def test_backward(dy_type, x_type, dx_type, dev):
    for i, (M, K) in enumerate(SIZES):
        shift, w_type = (0, 0, 1, 4)[i % 4], TYPES[i % 2]
        say("layer norm backward", M, K, dy_type, x_type, dx_type, w_type, shift)
        x, w, _, dy = _inputs(M, K, 200 + K, w_type, i % 5 != 3)
        _check_backward(*_backward(dev, dy, x, w, dy_type, x_type, w_type, dx_type, shift), dx_type)


@pytest.mark.parametrize("M,K", [(1025, 75), (2100, 264), (777, 2048), (300, 4096), (64, 16400)])
def test_many_rows(M, K, dev):
    """More rows than the launch has workgroups, and a last chunk that is not full."""
    say("layer norm rows", M, K)
    x, w, b, dy = _inputs(M, K, 300 + K, "f32")
    _check_forward(*_forward(dev, x, w, b, "f32", "bf16", "bf16"), "bf16")
    _check_backward(*_backward(dev, dy, x, w, "bf16", "f32", "bf16", "f32"), "f32")


@pytest.mark.parametrize("dy_type,x_type", list(itertools.product(TYPES, TYPES)))
@pytest.mark.parametrize("M,K,shift", [(1, 8193, 0), (2, 8200, 1), (3, 9445, 0), (600, 8195, 3), (2, 16383, 0), (3, 16384, 1)])
def test_odd_rows_in_sixteen_waves(M, K, shift, dy_type, x_type, dev):
    """Rows between 8192 and 16384 that no 16-byte access can take."""
    say("odd rows", M, K, shift, dy_type, x_type)
    x, w, b, dy = _inputs(M, K, 600 + K, "f32")
    _check_forward(*_forward(dev, x, w, b, x_type, "bf16", dy_type, shift), dy_type)
    _check_backward(*_backward(dev, dy, x, w, dy_type, x_type, "f32", x_type, shift), x_type)
    _check_backward(*_backward(dev, dy, x, None, dy_type, x_type, "f32", x_type, shift, (False, True, True)), x_type)
    _check_backward(*_backward(dev, dy, x, w, dy_type, x_type, "f32", x_type, shift, (True, False, False)), x_type)


@pytest.mark.parametrize("want", [w for w in itertools.product((True, False), repeat=3) if any(w)])
def test_each_output_is_optional(want, dev):
    say("outputs", want)
    for M, K in ((5, 2048), (70, 75), (3, 16400)):
        x, w, _, dy = _inputs(M, K, 400 + K, "f32")
        _check_backward(*_backward(dev, dy, x, w, "f32", "f32", "f32", "f32", want=want), "f32")


@pytest.mark.parametrize("M,K", [(4, 75), (70, 2048), (3, 4096), (2, 16400)])
@pytest.mark.parametrize("kind", TYPES)
def test_in_place_has_the_bits_of_the_call_into_another_buffer(M, K, kind, dev):
    import torch
    say("in place", M, K, kind)
    x, w, b, dy = _inputs(M, K, 500 + K, "f32")
    xt, wt, bt, dyt = put(x, kind, dev), put(w, "f32", dev), put(b, "f32", dev), put(dy, kind, dev)
    y, mean, rstd = torch.empty_like(xt), *(torch.empty(M, device=dev) for _ in range(2))
    H.hydra_layer_norm(xt, wt, bt, y, mean, rstd)
    x2 = xt.clone()
    H.hydra_layer_norm(x2, wt, bt, x2)
    assert torch.equal(x2, y)
    out = [torch.empty_like(xt), torch.empty(K, device=dev), torch.empty(K, device=dev)]
    H.hydra_layer_norm_backward(dyt, xt, wt, mean, rstd, *out)
    for over in ("dy", "x"):
        a = {"dy": dyt.clone(), "x": xt.clone()}
        dw, db = torch.empty(K, device=dev), torch.empty(K, device=dev)
        H.hydra_layer_norm_backward(a["dy"], a["x"], wt, mean, rstd, a[over], dw, db)
        assert torch.equal(a[over], out[0]) and torch.equal(dw, out[1]) and torch.equal(db, out[2]), over


def test_values_far_from_zero_and_constant_rows(dev):
    """The variance comes from centred values: a mean of a thousand times the width costs nothing but the mean's own
    rounding; a constant row gives the bias."""
    for K in (64, 2048, 4099, 16400):
        say("far from zero", K)
        r = np.random.default_rng(K)
        x = np.stack([1000 + r.normal(0, 1, K), np.full(K, 3.25), -1e4 + r.normal(0, 5, K), np.zeros(K)])
        v, y, mean, rstd = _forward(dev, x, r.normal(1, 0.2, K), r.normal(0, 1, K), "f32", "f32", "f32")
        _check_forward(v, y, mean, rstd, "f32")
        near(f64(y)[1], v[2], 1e-6 + 0 * v[2], "constant row")
        assert np.array_equal(f64(y)[3], v[2])
        v, y, mean, rstd = _forward(dev, x * 1e-4, None, None, "f32", "f32", "f32", eps=1e-12)
        _check_forward(v, y, mean, rstd, "f32", 1e-12)


@pytest.mark.parametrize("K", [75, 2048, 4096, 16400])
def test_bad_values_stay_in_their_row(K, dev):
    import torch
    say("bad rows", K)
    x, w, b, dy = _inputs(6, K, 600 + K, "f32")
    x[1, K // 2], x[3, 0], x[4, K - 1] = np.nan, np.inf, -np.inf
    v, y, mean, rstd = _forward(dev, x, w, b, "f32", "f32", "bf16")
    good, bad = [0, 2, 5], [1, 3, 4]
    assert np.isnan(f64(y)[bad]).all() and np.isnan(f64(rstd)[bad]).all()
    ref, tol = layer_norm_ref(v[0][good], v[1], v[2]), norm_bounds(v[0][good], v[1], v[2], "bf16")
    near(f64(y)[good], ref[0], tol[0], "y")
    xt, dyt = put(x, "f32", dev), put(dy, "f32", dev)
    dx, dw = torch.empty_like(xt), torch.empty(K, device=dev)
    H.hydra_layer_norm_backward(dyt, xt, put(w, "f32", dev), mean, rstd, dx, dw)
    assert np.isnan(f64(dx)[bad]).all() and np.isfinite(f64(dx)[good]).all() and np.isnan(f64(dw)).all()


@pytest.mark.parametrize("M", [3, 300])
def test_sums_at_any_alignment(M, dev):
    """dweight and dbias need 4-byte alignment alone, also where the rows are read 16 bytes at a time."""
    import torch
    for K in (264, 2048, 4096, 12000):
        say("sums at any alignment", M, K)
        x, w, _, dy = _inputs(M, K, 700 + K, "f32")
        v, (dx, dw, db) = _backward(dev, dy, x, w, "bf16", "bf16", "bf16", "bf16")
        flat = torch.full((2 * K + 16,), 7.0, device=dev)
        dw2, db2 = flat[1:K + 1], flat[K + 3:2 * K + 3]
        dx2 = torch.empty_like(dx)
        H.hydra_layer_norm_backward(put(dy, "bf16", dev), put(x, "bf16", dev), put(w, "bf16", dev), put(v[3], "f32", dev),
                                    put(v[4], "f32", dev), dx2, dw2, db2)
        assert torch.equal(dx2, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)
        assert (flat[[0, K + 1, K + 2]] == 7).all() and (flat[2 * K + 3:] == 7).all()


def test_repeated_calls_give_the_same_bits(dev):
    import torch
    x, w, _, dy = _inputs(700, 2048, 7, "f32")
    runs = [_backward(dev, dy, x, w, "bf16", "bf16", "bf16", "bf16")[1] for _ in range(3)]
    for o in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, runs[0]))
