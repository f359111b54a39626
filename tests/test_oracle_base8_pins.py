"""Pins of the 8-bit base's oracle against things other than itself: torch's own 8-bit type, closed forms, published test
vectors, exact distributions, differences, and planted mistakes."""
import numpy as np
import pytest
import torch

from oracle import base8_oracle as O


def test_codes_are_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3_values(), t, equal_nan=True)


def test_rounding_is_torchs():
    r = np.random.default_rng(0)
    v = np.concatenate([r.uniform(-448, 448, 4000), r.normal(0, 1e-2, 4000), O.VALUES[:127],
                        (O.VALUES[1:127] + O.VALUES[:126]) / 2, [2.0 ** -10, 2.0 ** -10 * 1.001, 448.0]])
    v = v.astype(np.float32).astype(np.float64)
    assert np.array_equal(O._round(v), torch.tensor(v).float().to(torch.float8_e4m3fn).double().numpy())


@pytest.mark.parametrize("rows", [1, 128])
def test_scales_are_the_least_that_fit(rows):
    r = np.random.default_rng(1)
    x = r.normal(0, 1, (200, 300)) * np.exp2(r.integers(-40, 40, (200, 1)))
    x[5] = 0
    q, e = O.quantize_ref(x, rows)
    for i in range(e.shape[0]):
        for j in range(e.shape[1]):
            b = np.abs(x[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128])
            assert b.max() <= 448 * 2.0 ** e[i, j]
            assert e[i, j] == -127 or b.max() > 448 * 2.0 ** (e[i, j] - 1)
    # half a step: 2^-4 of a value, or half the least step of the block's scale
    scale = np.repeat(np.repeat(2.0 ** e, rows, 0)[:200], 128, 1)[:, :300]
    assert np.all(np.abs(O.dequantize_ref(q, e, rows) - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * scale))


def test_borders_of_a_scale():
    for a, e in ((448.0, 0), (448.0000001, 1), (224.0, -1), (1.75, -8), (2.0, -7), (0.0, -127), (2.0 ** -140, -127)):
        assert O.quantize_ref([[a]], 1)[1][0, 0] == e, a
    q, e = O.quantize_ref([[np.inf, 1.0, np.nan, -np.inf]], 1)
    assert e[0, 0] == -8 and np.array_equal(np.isnan(q[0]), [True, False, True, True])


def test_a_tile_and_its_transpose_are_one():
    x = np.random.default_rng(2).normal(0, 1, (150, 260))
    q, e = O.quantize_ref(x, 128)
    qt, et = O.quantize_ref(x.T, 128)
    assert np.array_equal(q.T, qt) and np.array_equal(e.T, et)


def test_philox_known_answers():
    """The published vectors of philox4x32-10."""
    f = 0xFFFFFFFF
    assert O.philox_ref((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert O.philox_ref((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert O.philox_ref((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [
        0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_bits_by_element():
    b = O.dropout_bits_ref(7, 9, np.arange(16))
    w = O.philox_ref((1, 0, 9, 0), (7, 0))
    assert [b[8 + 2 * j] + (b[9 + 2 * j] << 16) for j in range(4)] == w
    assert np.array_equal(O.dropout_bits_ref(-1, 0, [0]), O.dropout_bits_ref((1 << 64) - 1, 0, [0]))
    f = O.dropout_factor_ref(3, 4, 0.25, (40, 50))
    assert set(np.unique(f)) == {0.0, 4 / 3} and abs(f.mean() - 1) < 5 * np.sqrt(1 / 3 / 2000)
    assert np.all(O.dropout_factor_ref(3, 4, 0.0, (9,)) == 1) and np.all(O.dropout_factor_ref(3, 4, 1.0, (9,)) == 0)


def _differences(backward):
    """The largest difference of the gradients from central differences of sum(dy * y) in the values (the function is
    linear in each argument, so that differences are exact but for rounding)."""
    r = np.random.default_rng(3)
    M, N, K, R, s = 3, 4, 5, 2, 1.7
    x, W, A, B, dy = (r.normal(0, 1, d) for d in ((M, K), (N, K), (R, K), (N, R), (M, N)))
    factor = O.dropout_factor_ref(1, 2, 0.4, (M, K))

    def f():
        return (dy * (x @ W.T + s * ((x * factor) @ A.T) @ B.T)).sum()

    got = backward(x * factor, W, A, B, s, dy, factor, quantize=False)
    worst = 0.0
    for a, g in zip((x, A, B), got):
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + 1e-3
            up = f()
            a[i] = keep - 1e-3
            dn = f()
            a[i] = keep
            worst = max(worst, abs((up - dn) / 2e-3 - g[i]))
    return worst


def test_gradients_by_differences():
    assert _differences(O.fp8_linear_backward_ref) < 1e-10


def test_planted_mistakes_in_the_gradients_are_found():
    def no_mask(xa, W, A, B, s, dy, factor, quantize):
        return O.fp8_linear_backward_ref(xa, W, A, B, s, dy, None, quantize)

    def no_scale(xa, W, A, B, s, dy, factor, quantize):
        return O.fp8_linear_backward_ref(xa, W, A, B, 1.0, dy, factor, quantize)

    def mask_on_the_base(xa, W, A, B, s, dy, factor, quantize):
        dx, dA, dB = O.fp8_linear_backward_ref(xa, W, A, B, s, dy, None, quantize)
        return dx * factor, dA, dB

    for f in (no_mask, no_scale, mask_on_the_base):
        assert _differences(f) > 1e-2


def _emitted(p, q, verify):
    """The exact distribution of the first token that comes out for one draft: over every draft, by the share of u that
    accepts it (bisection), and over every next token, by the shares of the second u (a fine grid's borders)."""
    V = len(p)
    with np.errstate(divide="ignore"):
        z, zd = np.log(p), np.log(q)
    out = np.zeros(V)
    target = np.stack([z, z])[None]
    for t in range(V):
        if q[t] == 0:
            continue
        grid = (np.arange(4000) + 0.5) / 4000
        for u in (grid[::40]):
            acc, tok, _, _ = verify(target, zd[None, None], [[t]], None, np.array([[u, 0.5]]))
            if acc[0] == 1:
                out[tok[0, 0]] += q[t] / 100
                continue
            for v in grid[::40]:
                out[verify(target, zd[None, None], [[t]], None, np.array([[u, v]]))[1][0, 0]] += q[t] / 100 / 100
    return out


def test_emitted_tokens_follow_the_target():
    p = np.array([0.4, 0.1, 0.3, 0.15, 0.05])
    for q in (np.array([0.1, 0.5, 0.2, 0.0, 0.2]), p):
        assert np.abs(_emitted(p, q, O.verify_ref) - p).max() < 0.011  # (a hundred values of each u)


def test_a_planted_mistake_in_the_verification_is_found():
    def from_p(target, draft, drafts, lens, u):  # a rejected position sampled from p instead of what p has left
        acc, tok, lp, odd = O.verify_ref(target, draft, drafts, lens, u)
        if acc[0] == 0:
            tok = O.verify_ref(target[:, :1], None, [[]], None, u[:, 1:])[1]
        return acc, tok, lp, odd

    p, q = np.array([0.4, 0.1, 0.3, 0.15, 0.05]), np.array([0.1, 0.5, 0.2, 0.0, 0.2])
    assert np.abs(_emitted(p, q, from_p) - p).max() > 0.05


def test_verification_closed_forms():
    z = np.log(np.array([[0.5, 0.25, 0.25], [0.2, 0.3, 0.5], [1e-9, 1.0, 1e-9]]))[None]
    u = np.array([[0.4, 0.9, 0.0]])
    # no distribution of the draft: accepted with p(t); the second is not (0.9 >= 0.3), and is left out
    acc, tok, lp, odd = O.verify_ref(z, None, [[0, 1]], None, u)
    assert acc[0] == 1 and tok.tolist() == [[0, 0, -1]] and not odd
    assert np.allclose(lp, np.log([[0.5, 0.2, 1.0]]))
    u[0, 2] = 0.3  # of 0.7: past 0.2
    assert O.verify_ref(z, None, [[0, 1]], None, u)[1].tolist() == [[0, 2, -1]]
    u[0, 1] = 0.1
    assert O.verify_ref(z, None, [[0, 1]], None, u)[1].tolist() == [[0, 1, 1]]
    assert O.verify_ref(z, None, [[0, 1]], [0], u)[1].tolist() == [[0, -1, -1]]
    # temperature: p ~ (4, 1, 1) at T = 1/2
    lp = O.verify_ref(z[:, :1], None, [[]], None, np.array([[0.0]]), 0.5)[2]
    assert np.isclose(lp[0, 0], np.log(4 / 6))
    # a draft that cannot be one, a row without a distribution
    acc, tok, lp, odd = O.verify_ref(z, None, [[3, 1]], None, u)
    assert acc[0] == 0 and tok[0, 0] == 0 and odd
    z[0, 1, 0] = np.nan
    acc, tok, lp, odd = O.verify_ref(z, None, [[0, 1]], None, u)
    assert acc[0] == 1 and tok.tolist() == [[0, -1, -1]] and np.isnan(lp[0, 1]) and odd
