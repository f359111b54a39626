"""hydra_dropout against the oracle's generator, bit for bit: types, residuals, lengths and alignments that meet every
path, p from 0 to 1, elements that are not finite, in place, far offsets, the same mask in the backward, graphs."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import dropout_bits_ref, dropout_factor_ref
from gpu_helpers import say
from base8_helpers import f64, put, rng_of

pytestmark = pytest.mark.gpu

TYPES = ("bf16", "f32")
SEED, OFFSET = -0x123456789ABCDEF, 0x1F2345678


def expected(x, factor, res, y_type):
    """fp32 product and sum, each rounded once, then the type."""
    import torch
    v = np.where(factor != 0, x.astype(np.float32) * np.float32(factor.max() if factor.any() else 0), np.float32(0))
    if res is not None:
        v = (v + res.astype(np.float32)).astype(np.float32)
    t = torch.tensor(v)
    return f64(t.to(torch.bfloat16) if y_type == "bf16" else t)


@pytest.mark.parametrize("n", [1, 7, 8, 9, 2048, 5003])
@pytest.mark.parametrize("xt", TYPES)
@pytest.mark.parametrize("rt", (None,) + TYPES)
@pytest.mark.parametrize("yt", TYPES)
def test_dropout(dev, n, xt, rt, yt):
    import torch
    say("dropout", n, xt, rt, yt)
    r = np.random.default_rng(n)
    x = put(r.normal(0, 1, n), xt, dev)
    res = None if rt is None else put(r.normal(0, 3, n), rt, dev)
    factor = dropout_factor_ref(SEED, OFFSET, 0.3, (n,))
    ref = expected(f64(x), factor, None if res is None else f64(res), yt)
    for shift in (0, 1):  # (the second: off the 16-byte boundaries)
        y = put(np.full(n, np.nan), yt, dev, shift=shift)
        H.hydra_dropout(x, y, 0.3, rng_of(SEED, OFFSET, dev), residual=res)
        torch.cuda.synchronize()
        assert np.array_equal(f64(y), ref)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -18, 2.0 ** -16, 0.05, 0.5, 1 - 2.0 ** -16, 1.0])
def test_probabilities(dev, p):
    import torch
    n = 4096
    x = put(np.random.default_rng(1).normal(0, 1, n), "f32", dev)
    y = torch.empty_like(x)
    H.hydra_dropout(x, y, p, rng_of(5, 6, dev))
    torch.cuda.synchronize()
    assert np.array_equal(f64(y), expected(f64(x), dropout_factor_ref(5, 6, p, (n,)), None, "f32"))


def test_dropped_elements_do_not_count(dev):
    import torch
    n = 1000
    factor = dropout_factor_ref(1, 2, 0.5, (n,))
    x = np.random.default_rng(2).normal(0, 1, n)
    x[0::3], x[1::3] = np.nan, np.inf
    y = torch.empty(n, device=dev)
    H.hydra_dropout(put(x, "f32", dev), y, 0.5, rng_of(1, 2, dev))
    got = f64(y)
    assert np.all(got[factor == 0] == 0)
    assert np.array_equal(np.isnan(got), (factor != 0) & np.isnan(x)) and np.array_equal(np.isinf(got), (factor != 0) & np.isinf(x))


def test_in_place_and_over_the_residual(dev):
    import torch
    r = np.random.default_rng(3)
    a, b = r.normal(0, 1, (33, 40)), r.normal(0, 1, (33, 40))
    rng = rng_of(3, 4, dev)
    ref = torch.empty((33, 40), device=dev)
    H.hydra_dropout(put(a, "f32", dev), ref, 0.2, rng, residual=put(b, "f32", dev))
    x, res = put(a, "f32", dev), put(b, "f32", dev)
    H.hydra_dropout(x, x, 0.2, rng, residual=res)
    assert torch.equal(x, ref)
    x = put(a, "f32", dev)
    H.hydra_dropout(x, res, 0.2, rng, residual=res)
    assert torch.equal(res, ref)


def test_seeds_and_offsets_are_64_bits(dev):
    import torch
    x = torch.ones(64, device=dev)
    y = torch.empty_like(x)
    for seed, offset in ((0, 0), (1 << 40, 0), (0, 1 << 40), (-1, -1), ((1 << 63) - 1, -(1 << 63))):
        H.hydra_dropout(x, y, 0.5, rng_of(seed, offset, dev))
        torch.cuda.synchronize()
        assert np.array_equal(f64(y), dropout_factor_ref(seed, offset, 0.5, (64,)))


def test_indices_past_32_bits(dev):
    """The last elements of a tensor of more than 2^35 / 8 elements: their blocks' numbers, and the addresses."""
    import torch
    n = (1 << 32) + 24
    x = torch.ones(n, dtype=torch.bfloat16, device=dev)
    H.hydra_dropout(x, x, 0.5, rng_of(11, 12, dev))
    torch.cuda.synchronize()
    for lo in (0, (1 << 31) - 16, (1 << 32) - 16, n - 16):
        bits = dropout_bits_ref(11, 12, np.arange(lo, lo + 16))
        assert np.array_equal(f64(x[lo:lo + 16]), np.where(bits >= 32768, 2.0, 0.0)), lo
    del x


def test_backward_is_the_same_mask(dev):
    """The gradient of sum(dy * dropout(x)), against the formula and against differences."""
    import torch
    r = np.random.default_rng(7)
    n = 520
    rng = rng_of(8, 9, dev)
    x, dy = put(r.normal(0, 1, n), "f32", dev), put(r.normal(0, 1, n), "f32", dev)
    dx, up, dn = (torch.empty_like(x) for _ in range(3))
    H.hydra_dropout(dy, dx, 0.1, rng)
    factor = dropout_factor_ref(8, 9, 0.1, (n,))
    assert np.array_equal(f64(dx), expected(f64(dy), factor, None, "f32"))
    H.hydra_dropout(x + 0.5, up, 0.1, rng)
    H.hydra_dropout(x - 0.5, dn, 0.1, rng)
    diff = (f64(up) - f64(dn)) * f64(dy)
    # x +- 1/2 and the two products are rounded: 4 half steps of values below 6
    assert np.all(np.abs(diff - f64(dx)) <= 4 * 2.0 ** -24 * 6 * np.abs(f64(dy)) + 2.0 ** -24 * np.abs(f64(dx)))


def test_a_replayed_graph_draws_new_masks(dev):
    import torch
    x, y = torch.ones(1 << 14, device=dev), torch.empty(1 << 14, device=dev)
    rng, one = rng_of(21, 0, dev), torch.tensor([0, 1], dtype=torch.int64, device=dev)
    H.hydra_dropout(x, y, 0.5, rng)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        H.hydra_dropout(x, y, 0.5, rng)
        rng.add_(one)
    masks = []
    for k in range(4):
        g.replay()
        torch.cuda.synchronize()
        masks.append(f64(y))
        e = torch.empty_like(x)
        H.hydra_dropout(x, e, 0.5, rng_of(21, k, dev))
        torch.cuda.synchronize()
        assert np.array_equal(masks[-1], f64(e))
    # independent masks agree in half the places: 2^14 of them, 6 sigma
    for a in range(4):
        for b in range(a):
            assert abs((masks[a] == masks[b]).mean() - 0.5) < 6 * 0.5 / 128


def test_shapes_that_differ_are_refused(dev):
    import torch
    x, rng = torch.ones(4, 8, device=dev), rng_of(0, 0, dev)
    with pytest.raises(ValueError):
        H.hydra_dropout(x, torch.empty(8, 4, device=dev), 0.1, rng)
    with pytest.raises(ValueError):
        H.hydra_dropout(x, torch.empty_like(x), 0.1, rng, residual=torch.empty(4, 7, device=dev))
    with pytest.raises(ValueError):
        H.hydra_dropout(x.t(), torch.empty(8, 4, device=dev), 0.1, rng)
    with pytest.raises(TypeError):
        H.hydra_dropout(x, torch.empty_like(x), 0.1, torch.zeros(2, device=dev))
    with pytest.raises(ValueError):
        H.hydra_dropout(x, torch.empty_like(x), 0.1, torch.zeros(3, dtype=torch.int64, device=dev))
    with pytest.raises(H.HydraError):
        H.hydra_dropout(x, torch.empty_like(x), 1.5, rng)
