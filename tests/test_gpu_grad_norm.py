"""The norm over many gradient tensors and the clipped gradients against the float64 oracle: sizes, counts, alignments,
both types, in place and into other buffers, values whose squares leave the range of fp32."""
import itertools

import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import grad_clip_ref, grad_norm_ref
from gpu_helpers import say
from update_helpers import TYPES, U, empty, f64, near, out_step, put

pytestmark = pytest.mark.gpu

SIZES = [1, 2, 3, 5, 8, 63, 64, 65, 1000, 4096, 16383, 16384, 16385, 33000, 100003]


def _tensors(dev, sizes, kinds, seed=0, std=1.0, shifts=(0, 1, 2, 3, 4, 7)):
    r = np.random.default_rng(seed)
    return [put(r.normal(0, std, n), kinds[i % len(kinds)], dev, shifts[i % len(shifts)]) for i, n in enumerate(sizes)]


def _clip(dev, grads, max_norm, outs=None):
    import torch
    norm, err = empty(1, "f32", dev), torch.zeros(1, dtype=torch.int32, device=dev)
    H.hydra_grad_clip(grads, max_norm, norm, outs, err_flag=err)
    return f64(norm)[0], err.item()


def _check(got, ref, kind, what):
    """The coefficient and the product are rounded once each, then the type."""
    near(f64(got), ref, (2.5 * U + (out_step(kind) * (1 + 2 ** -8) if kind == "bf16" else 0)) * np.abs(ref) + 1e-40, what)


@pytest.mark.parametrize("kinds", [("f32",), ("bf16",), ("f32", "bf16", "bf16")])
@pytest.mark.parametrize("sizes", [[1], [7], [16384], [50001], SIZES, [3] * 130, [2048] * 300, [0, 5, 0, 0, 9]])
def test_norm(sizes, kinds, dev):
    say("grad norm", len(sizes), sizes[0], kinds)
    grads = _tensors(dev, sizes, kinds, len(sizes))
    norm = empty(1, "f32", dev)
    H.hydra_grad_norm(grads, norm)
    ref = grad_norm_ref([f64(g) for g in grads])
    near(f64(norm), [ref], 1.5 * U * ref, "norm")
    got, err = _clip(dev, [g.clone() for g in grads], float("inf"))
    assert got == f64(norm)[0] and err == 0


@pytest.mark.parametrize("kind,out_kind", list(itertools.product(TYPES, TYPES)))
@pytest.mark.parametrize("max_norm", [0.25, 1e9, 0.0])
def test_clip_into_other_buffers(kind, out_kind, max_norm, dev):
    import torch
    say("clip", kind, out_kind, max_norm)
    grads = _tensors(dev, SIZES, (kind,), 5)
    flat = torch.full((sum(SIZES) + 7,), 9.0, device=dev, dtype=empty(1, out_kind, dev).dtype)
    outs = list(flat[:sum(SIZES)].split(SIZES))  # views at any alignment, side by side
    v = [f64(g) for g in grads]
    norm, err = _clip(dev, grads, max_norm, outs)
    ref, scaled = grad_clip_ref(v, max_norm)
    near([norm], [ref], 1.5 * U * ref, "norm")
    for o, s, n in zip(outs, scaled, SIZES):
        _check(o, s, out_kind, f"out {n}")
    assert err == 0 and (flat[sum(SIZES):] == 9).all()
    for g, a in zip(grads, v):
        assert np.array_equal(f64(g), a)  # the gradients themselves stay


@pytest.mark.parametrize("kind,out_kind", list(itertools.product(TYPES, TYPES)))
def test_clip_at_any_alignment(kind, out_kind, dev):
    """Gradients and results that lie apart to 16-byte boundaries; what lies around the results is left as it was."""
    import torch
    say("clip alignments", kind, out_kind)
    for n in (5, 9001):
        a = np.random.default_rng(n).normal(0, 1, n)
        for shift, out_shift in itertools.product(range(8), range(8)):
            g = put(a, kind, dev, shift)
            flat = torch.full((out_shift + n + 9,), 9.0, device=dev, dtype=empty(1, out_kind, dev).dtype)
            out = flat[out_shift:out_shift + n]
            norm, err = _clip(dev, [g], 0.5, [out])
            ref, scaled = grad_clip_ref([f64(g)], 0.5)
            near([norm], [ref], 1.5 * U * ref, "norm")
            _check(out, scaled[0], out_kind, f"out {n} {shift} {out_shift}")
            out.fill_(9.0)
            assert err == 0 and (flat == 9).all()


@pytest.mark.parametrize("kinds", [("f32",), ("bf16",), ("f32", "bf16")])
@pytest.mark.parametrize("count", [1, 9, 130, 500])
def test_clip_in_place(kinds, count, dev):
    say("clip in place", kinds, count)
    sizes = (SIZES * 40)[:count] if count < 500 else [77 + i % 5 for i in range(count)]
    grads = _tensors(dev, sizes, kinds, 6)
    ref, scaled = grad_clip_ref([f64(g) for g in grads], 1.0)
    norm, err = _clip(dev, grads, 1.0)
    near([norm], [ref], 1.5 * U * ref, "norm")
    for i, (g, s) in enumerate(zip(grads, scaled)):
        _check(g, s, kinds[i % len(kinds)], f"tensor {i}")
    assert err == 0
    before = [g.clone() for g in grads]
    _clip(dev, grads, 1e9)  # below the limit nothing changes
    import torch
    assert all(torch.equal(a, b) for a, b in zip(before, grads))


@pytest.mark.parametrize("count", [900, 4096])
def test_many_tensors(count, dev):
    """Up to the most that a call takes: several launches of the sums and of the scaling."""
    import torch
    say("many tensors", count)
    gen = torch.Generator(device=dev)
    gen.manual_seed(count)
    sizes = [1 + (i * 37) % 300 for i in range(count)]
    flat = torch.randn(sum(sizes) + count, generator=gen, device=dev)
    grads, at = [], 0
    for n in sizes:  # one element apart: no two are one run
        grads.append(flat[at:at + n])
        at += n + 1
    v = torch.cat(grads).double().cpu()
    ref = float(v.square().sum().sqrt())
    ends = torch.tensor(sizes).cumsum(0) + torch.arange(count)  # the elements between
    between = flat[ends].clone()
    norm, err = _clip(dev, grads, 2.0)
    near([norm], [ref], 1.5 * U * ref, "norm")
    _check(torch.cat(grads), v.numpy() * (2.0 / ref), "f32", "clipped")
    assert err == 0 and torch.equal(flat[ends], between)


def test_the_same_outs_as_gradients_is_in_place(dev):
    import torch
    a = _tensors(dev, [1000, 70000, 3], ("f32", "bf16"), 8)
    b, c = [g.clone() for g in a], [g.clone() for g in a]
    _clip(dev, b, 2.0)
    _clip(dev, c, 2.0, list(c))
    assert all(torch.equal(x, y) for x, y in zip(b, c))
    d = [g.clone() for g in a]
    other = torch.empty_like(d[1])
    _clip(dev, d, 2.0, [d[0], other, d[2]])  # some in place, some not
    assert torch.equal(d[0], b[0]) and torch.equal(other, b[1]) and torch.equal(d[2], b[2]) and torch.equal(d[1], a[1])


@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e15, 1e25])
def test_squares_outside_the_range_of_fp32(scale, dev):
    say("range", scale)
    grads = _tensors(dev, [5000, 333], ("f32",), 9, std=scale)
    ref, scaled = grad_clip_ref([f64(g) for g in grads], 1e-3 * scale)
    norm, err = _clip(dev, grads, float(np.float32(1e-3 * scale)))
    near([norm], [ref], 1.5 * U * ref, "norm")
    for g, s in zip(grads, scaled):
        near(f64(g), s, 4 * U * np.abs(s) + 2e-45, "clipped")  # (below 1e-38 one step of a denormal)
    assert err == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_norm_that_is_not_finite_scales_nothing(bad, dev):
    import torch
    say("not finite", bad)
    grads = _tensors(dev, [1000, 20000, 9], ("f32", "bf16"), 10)
    grads[1][12345] = bad
    before = [g.clone() for g in grads]
    norm, err = _clip(dev, grads, 1.0)
    assert err == 1 and (np.isnan(norm) if np.isnan(bad) else norm == np.inf)
    assert all(torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) for a, b in zip(before, grads))
    big = [torch.full((100,), 3e38, device=dev)]  # finite gradients whose norm leaves fp32
    norm, err = _clip(dev, big, 1.0)
    assert norm == np.inf and err == 1 and (big[0] == 3e38).all()


def test_zeros(dev):
    grads = _tensors(dev, [100, 20000], ("f32",), 11, std=0.0)
    for limit in (0.0, 1.0):
        norm, err = _clip(dev, grads, limit)
        assert norm == 0 and err == 0 and all((g == 0).all() for g in grads)


def test_a_tensor_of_more_than_2_to_the_31_elements(dev):
    """2^31 + 5 bf16 elements (4 GiB): only the last ones are not zero."""
    import torch
    say("long tensor")
    n = (1 << 31) + 5
    g = torch.zeros(n, dtype=torch.bfloat16, device=dev)
    g[n - 3:] = 2.0
    g[0] = 2.0
    norm, _ = _clip(dev, [g], 1.0)
    assert norm == 4.0 and (g[n - 3:] == 0.5).all() and g[0] == 0.5 and g[n - 4] == 0


def test_results_do_not_depend_on_the_run(dev):
    import torch
    a = _tensors(dev, SIZES * 10, ("f32", "bf16"), 12)
    norms = set()
    for _ in range(3):
        b = [g.clone() for g in a]
        norms.add(_clip(dev, b, 1.0)[0])
    assert len(norms) == 1


@pytest.mark.parametrize("what,exc", [("host", ValueError), ("half", TypeError), ("strided", ValueError),
                                      ("outs_shape", ValueError), ("outs_count", ValueError), ("no_tensor", TypeError),
                                      ("twice", H.HydraError), ("none", H.HydraError), ("no_limit", TypeError)])
def test_refusals(what, exc, dev):
    import torch
    say("refusal", what)
    g = _tensors(dev, [64, 100], ("f32",), 13)
    keep = [t.clone() for t in g]
    norm = torch.full((1,), 7.0, device=dev)
    grads, outs, limit = list(g), None, 1.0
    if what == "host":
        grads[1] = grads[1].cpu()
    elif what == "half":
        grads[0] = grads[0].half()
    elif what == "strided":
        grads[1] = grads[1][::2]
    elif what == "outs_shape":
        outs = [torch.empty(64, device=dev), torch.empty(10, 10, device=dev)]
    elif what == "outs_count":
        outs = [torch.empty(64, device=dev)]
    elif what == "no_tensor":
        grads[0] = None
    elif what == "twice":
        grads = [g[0], g[1], g[0]]
    elif what == "none":
        grads = []
    elif what == "no_limit":
        limit = None
    with pytest.raises(exc):
        H.hydra_grad_clip(grads, limit, norm, outs)
    torch.cuda.synchronize()
    assert norm.item() == 7.0 and all(torch.equal(a, b) for a, b in zip(g, keep))
