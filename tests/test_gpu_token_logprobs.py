"""Token log-probabilities, entropy, alternatives and their gradient against the float64 oracle: both types, vocabularies
from one entry to the largest accepted, strides and alignments, masked rows, ties, NaN and infinities."""
import itertools

import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import token_logprobs_backward_ref, token_logprobs_ref
from gpu_helpers import say
from update_helpers import TYPES, U, empty, f64, logp_back_bounds, logp_bounds, near, put

pytestmark = pytest.mark.gpu
INF, LOW = float("inf"), float(np.finfo(np.float32).min)


def _logits(M, V, seed, std=2.0):
    return np.random.default_rng(seed).normal(0, std, (M, V))


def _forward(dev, z, tokens, top, kind, shift=0, stride=0, want_top_lp=True, workspace=None):
    import torch
    M, V = z.shape
    zt = put(z, kind, dev, shift, stride)
    tok = torch.as_tensor(np.asarray(tokens, np.int32)).to(dev)
    o = {k: empty(M, "f32", dev) for k in ("lp", "lse", "entropy")}
    o["ids"] = torch.full((M, top), -7, dtype=torch.int32, device=dev) if top else None
    o["top_lp"] = empty((M, top), "f32", dev) if top and want_top_lp else None
    o["err"] = torch.zeros(1, dtype=torch.int32, device=dev)
    H.hydra_token_logprobs(zt, tok, o["lp"], o["lse"], o["entropy"], o["ids"], o["top_lp"], workspace, o["err"])
    return zt, o


def _check(z, tokens, top, o, err=0):
    """z: the logits as stored."""
    ref = token_logprobs_ref(z, tokens, top)
    e_lse, e_h, e_lp = logp_bounds(z, ref)
    with np.errstate(invalid="ignore"):
        near(f64(o["lse"]), ref["lse"], np.nan_to_num(e_lse), "lse")
        near(f64(o["entropy"]), ref["entropy"], np.nan_to_num(e_h), "entropy")
        ok = [0 <= t < z.shape[1] for t in tokens]
        zt = np.array([z[m, t] if ok[m] else 0.0 for m, t in enumerate(tokens)])
        near(f64(o["lp"]), ref["lp"], np.nan_to_num(e_lp(zt), posinf=0.0), "lp")
        if top:
            assert np.array_equal(o["ids"].cpu().numpy(), ref["ids"]), "ids"
            if o["top_lp"] is not None:
                asked = np.take_along_axis(z, ref["ids"], 1)
                tol = np.stack([e_lp(asked[:, k]) for k in range(top)], 1)
                near(f64(o["top_lp"]), ref["top_lp"], np.nan_to_num(tol, posinf=0.0), "top_lp")
    assert o["err"].item() == err


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("M,V,top", [(1, 1, 0), (1, 1, 1), (2, 2, 2), (3, 5, 3), (2, 31, 31), (2, 33, 32), (5, 64, 8), (3, 255, 4),
                                     (2, 1000, 20), (4, 2047, 7), (2, 4096, 32), (3, 4099, 1), (2, 16384, 16), (1, 32000, 32),
                                     (6, 32000, 0), (3, 50272, 8), (2, 50273, 20), (1, 65537, 5), (1, 131072, 32),
                                     (1, 200003, 9)])
def test_sizes(M, V, top, kind, dev):
    say("token logprobs", M, V, top, kind)
    z = _logits(M, V, 10 + V + top)
    tokens = np.random.default_rng(V).integers(0, V, M)
    tokens[0], tokens[-1] = V - 1, 0
    for shift, stride in ((0, 0), (1, V + 3), (3, 0), (0, (V + 15) // 8 * 8)):
        zt, o = _forward(dev, z, tokens, top, kind, shift, stride)
        _check(f64(zt), tokens, top, o)


@pytest.mark.parametrize("kind", TYPES)
def test_largest_vocabulary(kind, dev):
    """2^21 entries: the extremes at the row's ends and among equals, checked against numpy."""
    V = 1 << 21
    say("largest vocabulary", kind)
    z = _logits(1, V, 3).astype(np.float32)
    z[0, V - 1], z[0, 0], z[0, 1234567] = 40, 40, 41
    zt, o = _forward(dev, z, [V - 1], 32, kind)
    zz = f64(zt)
    lse = 41 + np.log(np.exp(zz - 41).sum())
    near(f64(o["lse"]), [lse], 1e-4, "lse")
    near(f64(o["lp"]), [40 - lse], 1e-4, "lp")
    order = np.lexsort((np.arange(V), -zz[0]))[:32]
    assert list(order[:3]) == [1234567, 0, V - 1]
    assert np.array_equal(o["ids"].cpu().numpy()[0], order)


@pytest.mark.parametrize("M", [1, 2, 9, 40, 300, 1100])
def test_row_counts(M, dev):
    """From one row, which many workgroups share, to more rows than there are workgroups."""
    say("row counts", M)
    for V, top in ((5000, 5), (9001, 0)):
        z = _logits(M, V, M)
        tokens = np.random.default_rng(M).integers(0, V, M)
        zt, o = _forward(dev, z, tokens, top, "f32")
        _check(f64(zt), tokens, top, o)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V", [40, 1003, 32000, 70000])
def test_masked_rows(V, kind, dev):
    """Rows of which the mask leaves a few entries, one, none; masks of -inf and of the type's lowest value."""
    import torch
    say("masked rows", V, kind)
    low = float(torch.finfo(torch.bfloat16 if kind == "bf16" else torch.float32).min)
    z, r = _logits(9, V, V), np.random.default_rng(V + 1)
    for m, mask in enumerate((-INF, low)):
        z[m, r.random(V) < 0.9] = mask
        z[2 + m, np.arange(V) != V - 1] = mask
        z[4 + m, :] = mask
    z[6, 5:], z[7, :V // 2], z[8, 3] = -INF, low, -INF
    tokens = np.array([0, V - 1, V - 1, V - 1, 2, 3, 4, V - 1, 3])
    zt, o = _forward(dev, z, tokens, 16, kind)
    _check(f64(zt), tokens, 16, o)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V", [64, 2050, 32000, 70001])
def test_ties_go_to_the_lowest_index(V, kind, dev):
    say("ties", V, kind)
    r = np.random.default_rng(V)
    z = np.zeros((7, V))
    z[1] = r.integers(0, 3, V)                     # three values
    z[2] = np.where(r.random(V) < 0.5, 0.0, -0.0)  # one value in two forms
    z[3] = np.sort(r.normal(0, 2, V))
    z[4] = -z[3]
    z[5] = r.integers(0, 40, V) / 8.0
    z[6, V // 2:] = 1.0                            # half a row of equals
    for top in (1, 8, 32):
        zt, o = _forward(dev, z, [0] * 7, top, kind)
        _check(f64(zt), [0] * 7, top, o)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V,shift,top", [(1, 0, 1), (40, 1, 32), (511, 0, 0), (1003, 3, 7), (2050, 0, 32), (4099, 2, 20),
                                         (10241, 0, 32), (10247, 5, 0), (12290, 0, 32), (16005, 1, 5), (19999, 0, 0)])
def test_rows_of_every_sort_many_times(V, shift, top, kind, dev):
    """Short rows in numbers: each sort against the oracle, its repetitions to the bit."""
    import torch
    say("rows many times", V, shift, top, kind)
    r = np.random.default_rng(V)
    z = r.normal(0, 2, (14, V))
    z[1], z[2], z[3] = 0.0, np.sort(z[2]), -np.sort(z[3])
    z[4, V // 2:], z[5, :], z[6, :] = -INF, -INF, LOW
    z[7, r.integers(0, V, max(1, V // 9))] = LOW
    z[8, :], z[8, V // 3] = LOW, 1.0
    z[9, V // 2], z[10, V - 1] = np.nan, INF
    z[11] = np.round(z[11])
    z[12] += 4.0e6
    z[13, ::2] = -INF
    tokens = list(r.integers(0, V, 13)) + [V]
    n = 64 if V < 3000 else 80 if V < 11000 else 32
    zt = put(np.tile(z, (n, 1)), kind, dev, shift, (V + 15) // 8 * 8)
    M = zt.shape[0]
    tok = torch.tensor(tokens * n, dtype=torch.int32, device=dev)
    o = {k: empty(M, "f32", dev) for k in ("lp", "lse", "entropy")}
    o["ids"] = torch.full((M, top), -7, dtype=torch.int32, device=dev) if top else None
    o["top_lp"] = empty((M, top), "f32", dev) if top else None
    o["err"] = torch.zeros(1, dtype=torch.int32, device=dev)
    H.hydra_token_logprobs(zt, tok, o["lp"], o["lse"], o["entropy"], o["ids"], o["top_lp"], None, o["err"])
    for k, v in o.items():
        if v is not None and k != "err":
            bits = v.view(torch.int32).view(n, 14, -1)
            assert (bits == bits[:1]).all(), k
            o[k] = v[:14]
    _check(f64(zt)[:14], tokens, top, o, err=1)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V", [33, 4000, 70000])
def test_nan_and_infinities(V, kind, dev):
    say("nan and infinities", V, kind)
    z = _logits(6, V, V)
    z[0, V // 3], z[1, 5], z[2, V - 1], z[2, 1] = np.nan, INF, INF, np.nan
    z[3, 7], z[4, :] = -INF, np.nan
    zt, o = _forward(dev, z, [1, 5, 1, 7, 0, 2], 12, kind)
    _check(f64(zt), [1, 5, 1, 7, 0, 2], 12, o)


def test_extreme_logits(dev):
    """Differences are formed first: logits of the type's largest and lowest values keep their meaning."""
    say("extreme logits")
    big = float(np.finfo(np.float32).max)
    z = np.array([[big, big, LOW, 0.0], [big, 0.9 * big, 0, 0], [-3e38, -3e38, LOW, LOW], [1e30, 1e30, 1e30, -1e30],
                  [2.5e38, 2.5e38, -2.5e38, 2.5e38]])
    zt, o = _forward(dev, z, [0, 1, 0, 2, 3], 4, "f32")
    _check(f64(zt), [0, 1, 0, 2, 3], 4, o)


@pytest.mark.parametrize("offset", [0, 2 ** 12, -2 ** 16, 2 ** 20, 2 ** 21, -2 ** 21, 2 ** 23, -2 ** 23])
@pytest.mark.parametrize("V", [600, 70000])
def test_common_offset(V, offset, dev):
    """A log-probability does not depend on what all logits of its row have in common: the difference to the rounded base
    is exact or off by U (d + 1), that to its rest by as much, that to ln s by U |lp|, whatever the offset is.  The logits
    are whole numbers, which fp32 holds with each offset; sorted, some segments lie on either side of it."""
    say("common offset", V, offset)
    z = np.random.default_rng(V).integers(-8, 0, (3, V)).astype(np.float64)
    z[1], z[2] = np.sort(z[1]), -np.sort(z[2])
    z[2, : V // 2] = -z[2, : V // 2]
    tokens = [V // 3, V - 1, 1]
    zt, o = _forward(dev, z + offset, tokens, 0, "f32")
    assert np.array_equal(f64(zt), z + offset)
    ref = token_logprobs_ref(z, tokens, 0)
    e_lse, e_h, _ = logp_bounds(z, ref)
    asked = np.take_along_axis(z, np.array(tokens)[:, None], 1)[:, 0]
    near(f64(o["lp"]), ref["lp"], e_lse + U * (2 * (z.max(1) - asked + 1) + np.abs(ref["lp"])), "lp")
    near(f64(o["entropy"]), ref["entropy"], e_h, "entropy")
    near(f64(o["lse"]), ref["lse"] + offset, e_lse + U * np.abs(ref["lse"] + offset), "lse")


def test_tokens_out_of_range(dev):
    say("tokens out of range")
    z = _logits(5, 100, 1)
    tokens = [0, -1, 100, 99, 2 ** 31 - 1]
    zt, o = _forward(dev, z, tokens, 3, "f32")
    _check(f64(zt), tokens, 3, o, err=1)


def test_outputs_are_optional(dev):
    import torch
    z = put(_logits(4, 3001, 2), "f32", dev)
    tok = torch.arange(4, dtype=torch.int32, device=dev)
    full = {k: torch.empty(4, device=dev) for k in ("lp", "lse", "entropy")}
    ids, tlp = torch.empty((4, 6), dtype=torch.int32, device=dev), torch.empty((4, 6), device=dev)
    H.hydra_token_logprobs(z, tok, full["lp"], full["lse"], full["entropy"], ids, tlp)
    for k in full:
        o = torch.full((4,), float("nan"), device=dev)
        H.hydra_token_logprobs(z, tok if k == "lp" else None, **{"lp": None, k: o})
        near(f64(o), f64(full[k]), 1e-5, k)
    ids2 = torch.full_like(ids, -1)
    H.hydra_token_logprobs(z, None, None, top_ids=ids2)
    assert torch.equal(ids, ids2)


# ---------------------------------------------------------------- gradient

def _backward(dev, z, tokens, d_lp, d_h, kind, d_kind, shift=0, stride=0, d_stride=0, d_shift=None):
    import torch
    M, V = z.shape
    zt = put(z, kind, dev, shift, stride)
    zz = f64(zt)
    fw = token_logprobs_ref(zz)
    t = {"lse": put(fw["lse"], "f32", dev), "d_lp": None if d_lp is None else put(d_lp, "f32", dev),
         "entropy": None if d_h is None else put(fw["entropy"], "f32", dev),
         "d_entropy": None if d_h is None else put(d_h, "f32", dev)}
    tok = None if tokens is None else torch.as_tensor(np.asarray(tokens, np.int32)).to(dev)
    dz = empty((M, V), d_kind, dev, shift if d_shift is None else d_shift, d_stride)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    H.hydra_token_logprobs_backward(zt, tok, t["lse"], dz, t["d_lp"], t["entropy"], t["d_entropy"], err)
    host = {k: None if v is None else f64(v) for k, v in t.items()}
    return zt, zz, host, dz, err


def _check_backward(zz, tokens, t, dz, d_kind):
    ref = token_logprobs_backward_ref(zz, tokens, t["lse"], t["d_lp"], t["entropy"], t["d_entropy"])
    near(f64(dz), ref, logp_back_bounds(zz, t["lse"], t["d_lp"], t["entropy"], t["d_entropy"], ref, d_kind), "d_logits")


@pytest.mark.parametrize("kind,d_kind", list(itertools.product(TYPES, TYPES)))
@pytest.mark.parametrize("M,V", [(1, 1), (2, 2), (3, 7), (4, 64), (5, 255), (3, 1000), (2, 4099), (7, 8192), (2, 32000),
                                 (3, 50272), (2, 50273), (1, 131080)])
def test_gradient(M, V, kind, d_kind, dev):
    say("gradient", M, V, kind, d_kind)
    r = np.random.default_rng(V)
    z, tokens = _logits(M, V, V + 1), r.integers(0, V, M)
    tokens[0], tokens[-1] = V - 1, 0
    d_lp, d_h = r.normal(0, 1, M), r.normal(0, 0.1, M)
    for i, (shift, stride, d_stride, d_shift) in enumerate(((0, 0, 0, 0), (1, 0, 0, 1), (0, V + 5, V + 9, 0), (3, V + 8, V, 2))):
        a, h = ((d_lp, None), (d_lp, d_h), (None, d_h), (d_lp, d_h))[i]
        zt, zz, t, dz, err = _backward(dev, z, None if a is None else tokens, a, h, kind, d_kind, shift, stride, d_stride, d_shift)
        _check_backward(zz, tokens, t, dz, d_kind)
        assert err.item() == 0


@pytest.mark.parametrize("kind,d_kind", list(itertools.product(TYPES, TYPES)))
def test_gradient_at_any_alignment(kind, d_kind, dev):
    """Rows and results that lie apart to 16-byte boundaries, and what lies around the results is left as it was."""
    import torch
    say("gradient alignments", kind, d_kind)
    M, V, ld = 3, 1061, 1070
    z, tokens, d_lp = _logits(M, V, 8), [1060, 0, 7], np.array([0.5, -1.0, 2.0])
    for shift, d_shift in itertools.product(range(8), range(8)):
        zt = put(z, kind, dev, shift, ld)
        zz = f64(zt)
        lse = put(token_logprobs_ref(zz)["lse"], "f32", dev)
        flat = torch.full((d_shift + M * ld + 8,), 7.0, dtype=empty(1, d_kind, dev).dtype, device=dev)
        dz = flat.as_strided((M, V), (ld, 1), d_shift)
        H.hydra_token_logprobs_backward(zt, torch.tensor(tokens, dtype=torch.int32, device=dev), lse, dz,
                                        put(d_lp, "f32", dev))
        _check_backward(zz, tokens, {"lse": f64(lse), "d_lp": d_lp, "entropy": None, "d_entropy": None}, dz, d_kind)
        dz.fill_(7.0)
        assert (flat == 7).all()


@pytest.mark.parametrize("kind", TYPES)
def test_rows_of_masked_entries_alone_have_no_gradient(kind, dev):
    """(NaN, as their log-probabilities; zeros where nothing is asked for; the rows beside them as ever)"""
    import torch
    say("rows of masked entries alone", kind)
    z = _logits(4, 3001, 3)
    z[1], z[2] = -INF, -INF
    zt = put(z, kind, dev)
    zz = f64(zt)
    lse = torch.tensor(token_logprobs_ref(zz)["lse"], dtype=torch.float32, device=dev)
    assert lse[1] == -INF
    d_lp, dz = np.array([1.0, 1.0, 0.0, -2.0]), empty((4, 3001), kind, dev)
    H.hydra_token_logprobs_backward(zt, torch.arange(4, dtype=torch.int32, device=dev), lse, dz, put(d_lp, "f32", dev))
    got = f64(dz)
    assert np.isnan(got[1]).all() and (got[2] == 0).all()
    live = [0, 3]
    ref = token_logprobs_backward_ref(zz[live], live, f64(lse)[live], d_lp[live])
    near(got[live], ref, logp_back_bounds(zz[live], f64(lse)[live], d_lp[live], None, None, ref, kind), "d_logits")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V", [75, 32000])
def test_rows_without_a_gradient_are_zeros(V, kind, dev):
    """Prompt tokens and padding: neither their logits nor their tokens count; elements past a row's end stay."""
    import torch
    say("rows without a gradient", V, kind)
    z = _logits(6, V, 9)
    d_lp = np.array([0.0, 1.5, -0.0, 0.0, -0.25, 0.0])
    zt = put(z, kind, dev, stride=V + 8)
    fw = token_logprobs_ref(f64(zt))
    zt[0, 3], zt[2, :], zt[5, 0] = float("nan"), float("inf"), float("-inf")
    lse = fw["lse"].copy()
    lse[[0, 2, 3, 5]] = np.nan
    tokens = torch.tensor([-100, 4, 2 ** 31 - 1, V, 0, -1], dtype=torch.int32, device=dev)
    wide = torch.full((6, V + 8), 7.0, device=dev, dtype=zt.dtype)
    err = torch.zeros(1, dtype=torch.int32, device=dev)
    H.hydra_token_logprobs_backward(zt, tokens, put(lse, "f32", dev), wide[:, :V], put(d_lp, "f32", dev), err_flag=err)
    got = f64(wide)
    assert np.all(got[[0, 2, 3, 5], :V] == 0) and np.all(got[:, V:] == 7) and err.item() == 0
    t = {"lse": f64(put(lse, "f32", dev)), "d_lp": f64(put(d_lp, "f32", dev)), "entropy": None, "d_entropy": None}
    live = [1, 4]
    t = {k: None if v is None else v[live] for k, v in t.items()}
    ref = token_logprobs_backward_ref(f64(zt)[live], [4, 0], t["lse"], t["d_lp"])
    near(got[live, :V], ref, logp_back_bounds(f64(zt)[live], t["lse"], t["d_lp"], None, None, ref, kind), "d_logits")


def test_token_out_of_range_in_the_gradient(dev):
    z = _logits(3, 50, 1)
    _, zz, t, dz, err = _backward(dev, z, [3, 50, -1], np.ones(3), None, "f32", "f32")
    got = f64(dz)
    assert np.isfinite(got[0]).all() and np.isnan(got[1:]).all() and err.item() == 1


@pytest.mark.parametrize("kind", TYPES)
def test_masked_entries_have_no_gradient(kind, dev):
    say("masked gradient", kind)
    z = _logits(4, 3000, 5)
    z[0, ::2], z[1, 1:], z[2, ::3] = -INF, -INF, LOW if kind == "f32" else -3e38
    tokens = [1, 0, 1, 7]
    d_lp, d_h = np.array([1.0, -2.0, 0.5, 0.0]), np.array([0.1, 0.2, -0.3, 1.0])
    _, zz, t, dz, _ = _backward(dev, z, tokens, d_lp, d_h, kind, "f32")
    _check_backward(zz, tokens, t, dz, "f32")
    assert np.all(f64(dz)[0, ::2] == 0) and np.all(f64(dz)[1] == 0)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V,stride", [(1000, 1000), (1003, 1003), (1000, 1012)])
def test_gradient_in_place(V, stride, kind, dev):
    """Into the logits themselves: the bits of the call into another buffer, entries past a row's end stay."""
    import torch
    say("gradient in place", V, stride, kind)
    r = np.random.default_rng(V)
    z, tokens, d_lp = _logits(9, V, V), r.integers(0, V, 9), r.normal(0, 1, 9) * (np.arange(9) % 3 > 0)
    zt, zz, t, dz, _ = _backward(dev, z, tokens, d_lp, r.normal(0, 0.1, 9), kind, kind, stride=stride, d_stride=stride)
    a = {k: put(v, "f32", dev) for k, v in t.items()}
    H.hydra_token_logprobs_backward(zt, torch.as_tensor(tokens.astype(np.int32)).to(dev), a["lse"], zt, a["d_lp"],
                                    a["entropy"], a["d_entropy"])
    assert torch.equal(zt, dz)
    if stride > V:
        assert torch.isnan(torch.as_strided(zt, (8, stride - V), (stride, 1), zt.storage_offset() + V)).all()


def test_gradient_against_differences_of_the_forward(dev):
    """Central differences of the library's own forward, on 12 logits: lp and H are known to 2e-6, a step of 0.02 leaves
    a third-order term of 0.02^2 / 6 times a third derivative below 2: 1.4e-4, and 2e-6 / 0.02 = 1e-4."""
    import torch
    say("differences")
    r = np.random.default_rng(3)
    z, d_lp, d_h = r.normal(0, 1, 12).astype(np.float32), 0.7, -0.4
    h = 0.02
    Z = np.concatenate([z + h * np.eye(12), z - h * np.eye(12)]).astype(np.float32)
    zt = torch.as_tensor(Z).to(dev)
    tok = torch.full((24,), 5, dtype=torch.int32, device=dev)
    lp, ent = torch.empty(24, device=dev), torch.empty(24, device=dev)
    H.hydra_token_logprobs(zt, tok, lp, entropy=ent)
    f = d_lp * f64(lp) + d_h * f64(ent)
    _, _, _, dz, _ = _backward(dev, z[None], [5], np.array([d_lp]), np.array([d_h]), "f32", "f32")
    near(f64(dz)[0], (f[:12] - f[12:]) / (2 * h), 4e-4, "gradient")


@pytest.mark.parametrize("kind,d_kind,M", [("f32", "f32", 700), ("f32", "bf16", 930), ("bf16", "f32", 930),
                                           ("bf16", "bf16", 1400)])
def test_gradient_larger_than_the_caches(kind, d_kind, M, dev):
    """Logits and gradient of more than 256 MB together go past the caches: the bits of the same rows in smaller calls,
    and a few rows against the oracle."""
    import torch
    say("large gradient", kind, d_kind, M)
    V = 50001  # (rows at every alignment)
    gen = torch.Generator(device=dev)
    gen.manual_seed(M)
    z = torch.randn(M, V, generator=gen, device=dev).to(empty(1, kind, dev).dtype)
    tok = torch.randint(0, V, (M,), generator=gen, device=dev, dtype=torch.int32)
    lse, d_lp = torch.logsumexp(z.float(), 1), torch.randn(M, generator=gen, device=dev)
    d_lp[::3] = 0
    dz = torch.full((M, V), float("nan"), device=dev, dtype=empty(1, d_kind, dev).dtype)
    assert z.numel() * (z.element_size() + dz.element_size()) > 1 << 28
    H.hydra_token_logprobs_backward(z, tok, lse, dz, d_lp)
    part = torch.empty_like(dz)
    for m in range(0, M, 280):
        r = slice(m, m + 280)
        H.hydra_token_logprobs_backward(z[r], tok[r], lse[r], part[r], d_lp[r])
    assert torch.equal(dz, part)
    rows = [0, 1, 2, M - 1]
    zz, t = f64(z[rows]), [f64(v[rows]) for v in (lse, d_lp)]
    ref = token_logprobs_backward_ref(zz, tok[rows].cpu().numpy(), *t)
    near(f64(dz[rows]), ref, logp_back_bounds(zz, t[0], t[1], None, None, ref, d_kind), "d_logits")


def test_rows_past_2_to_the_31_elements(dev):
    """Rows so far apart that their offsets leave 32 bits (a strided view of one large bf16 buffer)."""
    import torch
    say("far rows")
    V, ld, M = 5000, 1 << 30, 4  # 3 x 2 GiB apart
    buf = torch.empty((M - 1) * ld + V, dtype=torch.bfloat16, device=dev)
    z = buf.as_strided((M, V), (ld, 1))
    r = np.random.default_rng(0)
    z.copy_(torch.as_tensor(r.normal(0, 2, (M, V))))
    tokens = [0, 1, 4999, 77]
    o = {k: empty(M, "f32", dev) for k in ("lp", "lse", "entropy")}
    o["ids"], o["top_lp"] = torch.empty((M, 4), dtype=torch.int32, device=dev), empty((M, 4), "f32", dev)
    o["err"] = torch.zeros(1, dtype=torch.int32, device=dev)
    tok = torch.tensor(tokens, dtype=torch.int32, device=dev)
    H.hydra_token_logprobs(z, tok, o["lp"], o["lse"], o["entropy"], o["ids"], o["top_lp"], None, o["err"])
    zz = f64(z)
    _check(zz, tokens, 4, o)
    d_lp = put(np.ones(M), "f32", dev)
    H.hydra_token_logprobs_backward(z, tok, o["lse"], z, d_lp)
    ref = token_logprobs_backward_ref(zz, tokens, f64(o["lse"]), np.ones(M))
    near(f64(z), ref, logp_back_bounds(zz, f64(o["lse"]), np.ones(M), None, None, ref, "bf16"), "d_logits")
