"""Layer norm with more rows than a launch takes at once, and with more than 2^31 elements.

The forward launches at most 1024 workgroups of 4, 2 or 1 rows (up to 1024, 2048 and 4096 columns) and at most 512 of
one row (up to 16384): here each kind goes through a second or third round of rows, the last of them not full, with the
weights still in registers and the sums' LDS in use again."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import layer_norm_backward_ref, layer_norm_ref
from gpu_helpers import say
from test_gpu_layer_norm import _backward, _check_backward, _check_forward, _forward, _inputs
from update_helpers import TYPES, U, f64, near, norm_back_bounds, norm_bounds, put

pytestmark = pytest.mark.gpu

ROUNDS = [(4099, 264), (9001, 75), (4097, 1000), (2051, 2048), (5003, 1032), (2049, 2047), (1027, 4096), (2055, 2056),
          (1025, 4095), (515, 8192), (1030, 4104), (515, 8191), (515, 11008), (1026, 8200), (513, 16384), (514, 8193)]


@pytest.mark.parametrize("x_type,y_type", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("M,K", ROUNDS)
def test_forward_in_rounds(M, K, x_type, y_type, dev):
    import torch
    say("rounds of rows", M, K, x_type, y_type)
    x, w, b, _ = _inputs(M, K, 800 + K, "f32")
    v, y, mean, rstd = _forward(dev, x, w, b, x_type, "bf16", y_type)
    _check_forward(v, y, mean, rstd, y_type)
    if x_type == y_type:
        xt = put(x, x_type, dev)
        H.hydra_layer_norm(xt, put(w, "bf16", dev), put(b, "bf16", dev), xt)
        assert torch.equal(xt, y)


@pytest.mark.parametrize("dy_type,x_type", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("M,K", [(4099, 264), (2051, 2048), (2049, 2047), (1027, 4096), (515, 8192), (515, 11008),
                                 (514, 8193)])
def test_backward_in_rounds(M, K, dy_type, x_type, dev):
    say("rounds of rows, backward", M, K, dy_type, x_type)
    x, w, _, dy = _inputs(M, K, 900 + K, "f32")
    _check_backward(*_backward(dev, dy, x, w, dy_type, x_type, "f32", dy_type), dy_type)


@pytest.mark.parametrize("K,copies", [(2056, 256), (2049, 256), (16392, 32)])
def test_more_than_2_to_the_31_elements(K, copies, dev):
    """4096 rows over and over: every copy has the first one's bits, the first is held against the oracle.  A column's sum
    is 512 chains of M / 512 rows each and their 512 sums, or in rows past 16384 columns 16 chains of M / 16 rows (1024
    workgroups over 65 stretches of 256 columns) and their sums: no term passes through more additions than one chain's
    and one per chain."""
    import torch
    n = 4096
    M = n * copies
    assert M * K > 1 << 31
    say("many elements", M, K)
    gen = torch.Generator(device=dev)
    gen.manual_seed(K)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev).to(torch.bfloat16)

    one, d_one, w, b = normal(n, K) * 2 + 1, normal(n, K), normal(K), normal(K)
    x = one.repeat(copies, 1)
    y, mean, rstd = torch.empty_like(x), torch.empty(M, device=dev), torch.empty(M, device=dev)
    H.hydra_layer_norm(x, w, b, y, mean, rstd)

    def same(t):
        bits = t.view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).view(copies, -1)
        return all(torch.equal(bits[i], bits[0]) for i in range(copies))

    assert same(y) and same(mean) and same(rstd)
    rows = [0, 1, n // 2, n - 1]
    v = [f64(one[rows]), f64(w), f64(b)]
    ref, tol = layer_norm_ref(*v), norm_bounds(*v, "bf16")
    for got, r, t, what in zip((y, mean, rstd), ref, tol, ("y", "mean", "rstd")):
        near(f64(got[rows]), r, t, what)
    H.hydra_layer_norm(x, w, b, x)
    assert torch.equal(x, y)
    del y
    x.copy_(one.repeat(copies, 1))
    dy = d_one.repeat(copies, 1)
    dw, db = torch.empty(K, device=dev), torch.empty(K, device=dev)
    H.hydra_layer_norm_backward(dy, x, w, mean, rstd, dy, dw, db)
    assert same(dy)
    v = [f64(d_one[rows]), f64(one[rows]), f64(w), f64(mean[rows]), f64(rstd[rows])]
    near(f64(dy[rows]), layer_norm_backward_ref(*v)[0], norm_back_bounds(*v, "bf16")[0], "dx")
    xh = (one.double() - mean[:n, None].double()) * rstd[:n, None].double()
    each = d_one.double() * xh
    chains = 16 if K > 16384 else 512
    chain = U * (M / chains + chains)
    near(f64(dw), f64(each.sum(0) * copies), (chain + 4 * U) * f64(each.abs().sum(0) * copies), "dw")
    near(f64(db), f64(d_one.double().sum(0) * copies), chain * f64(d_one.double().abs().sum(0) * copies), "db")
