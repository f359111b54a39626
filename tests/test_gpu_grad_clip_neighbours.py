"""Gradient clipping where the norm and the flag stand right beside the gradients in one buffer, and lists of every
length around the launches' limits whose runs join and do not join."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import grad_clip_ref
from gpu_helpers import say
from update_helpers import U, f64, near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
def test_norm_and_flag_between_the_gradients(in_place, dev):
    import torch
    say("norm and flag between the gradients", in_place)
    values = np.random.default_rng(3).normal(0, 1, 3000).astype(np.float32)
    flat = torch.from_numpy(values).to(dev)
    g = [flat[:1000], flat[1001:2500], flat[2501:]]
    norm, flag = flat[1000:1001], flat[2500:2501].view(torch.int32)
    flag.zero_()
    outs = None if in_place else [torch.empty_like(t) for t in g]
    ref_norm, ref = grad_clip_ref([values[:1000], values[1001:2500], values[2501:]], 2.0)
    H.hydra_grad_clip(g, 2.0, norm, outs, err_flag=flag)
    near(f64(norm), [ref_norm], U * ref_norm * 2, "norm")
    assert flag.item() == 0
    # the factor is formed in 64 bits, rounded, and the product rounded
    for got, r in zip(g if in_place else outs, ref):
        near(f64(got), r, 3 * U * np.abs(r), "gradient")
    if not in_place:
        assert np.array_equal(f64(flat[:1000]), values[:1000].astype(np.float64))


@pytest.mark.parametrize("n", [1, 2, 175, 176, 177, 255, 256, 257, 352, 353, 512, 513, 4095, 4096])
def test_lists_around_the_launches_limits(n, dev):
    """Every third tensor stands apart from the one before it, every seventh is empty, types change along the list."""
    import torch
    say("lists", n)
    r = np.random.default_rng(n)
    kinds = [torch.float32 if (i // 5) % 2 else torch.bfloat16 for i in range(n)]
    sizes = [0 if i % 7 == 6 else int(r.integers(1, 90)) for i in range(n)]
    flat = torch.full((sum(sizes) * 4 + 16 * n,), float("nan"), device=dev)
    out = torch.full_like(flat, float("nan"))
    g, outs, at = [], [], 0
    for i, (kind, size) in enumerate(zip(kinds, sizes)):
        at += 8 if i % 3 == 0 else 0
        view = [b.view(kind) for b in (flat, out)]
        at += -at % (4 if kind == torch.float32 else 2)
        e = at // (4 if kind == torch.float32 else 2)
        g.append(view[0][e:e + size])
        outs.append(view[1][e:e + size])
        at += size * (4 if kind == torch.float32 else 2)
    for t in g:
        t.copy_(torch.from_numpy(r.normal(0, 1, t.numel()).astype(np.float32)))
    before = [f64(t) for t in g]
    norm, norm2 = torch.zeros(1, device=dev), torch.zeros(1, device=dev)
    H.hydra_grad_norm(g, norm2)
    H.hydra_grad_clip(g, 0.5, norm, outs)
    ref_norm, ref = grad_clip_ref(before, 0.5)
    near(f64(norm), [ref_norm], 2 * U * ref_norm, "norm")
    assert torch.equal(norm, norm2)
    for i in range(n):
        step = U if kinds[i] == torch.float32 else 2.0 ** -8
        near(f64(outs[i]), ref[i], (step + 3 * U) * np.abs(ref[i]) + 1e-40, f"gradient {i}")
    H.hydra_grad_clip(g, 0.5, norm)
    assert all(torch.equal(a, b) for a, b in zip(g, outs))
    # nothing between the tensors was written
    covered = torch.zeros_like(out, dtype=torch.bool).view(torch.uint8).repeat_interleave(4)
    for t in outs:
        if t.numel():
            lo = t.data_ptr() - out.data_ptr()
            covered[lo:lo + t.numel() * t.element_size()] = 1
    raw, nan = out.view(torch.uint8), torch.full_like(out, float("nan")).view(torch.uint8)
    assert torch.equal(raw[covered == 0], nan[covered == 0])
