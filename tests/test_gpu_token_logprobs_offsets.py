"""The gradient of log-probabilities and entropy of logits far from zero, against the float64 gradient of the logits
themselves.

The gradient goes by one fp32 lse, off by d = U |lse| (its rounding) and by what the forward's sum is off.  Every p_j is
then off by the factor e^d at most, and ln p_j by d: half a step of lse, 2.4e-4 at an offset of 4096, 0.06 at 2^20.  That
is the bound here, beside the one for a given lse."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import token_logprobs_backward_ref, token_logprobs_ref
from gpu_helpers import say
from update_helpers import U, empty, f64, logp_back_bounds, logp_bounds, near, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("offset", [0, 100, 2 ** 12, -2 ** 16, 2 ** 20, -2 ** 20])
@pytest.mark.parametrize("V", [7, 600, 50272])
def test_gradient_of_shifted_logits(V, offset, entropy, dev):
    import torch
    say("gradient of shifted logits", V, offset, entropy)
    r = np.random.default_rng(V)
    z = r.integers(-8, 8, (3, V)).astype(np.float64)   # (fp32 holds them with each offset)
    tokens, d_lp = [0, V // 2, V - 1], np.array([1.0, -0.5, 2.0])
    d_h = np.array([0.25, -0.125, 0.5]) if entropy else None
    zt, tok = put(z + offset, "f32", dev), torch.tensor(tokens, dtype=torch.int32, device=dev)
    assert np.array_equal(f64(zt), z + offset)
    lp, lse, h, dz = empty(3, "f32", dev), empty(3, "f32", dev), empty(3, "f32", dev), empty((3, V), "f32", dev)
    H.hydra_token_logprobs(zt, tok, lp, lse, h)
    H.hydra_token_logprobs_backward(zt, tok, lse, dz, put(d_lp, "f32", dev), h if entropy else None,
                                    put(d_h, "f32", dev) if entropy else None)
    fw = token_logprobs_ref(z, tokens)
    ref = token_logprobs_backward_ref(z, tokens, fw["lse"], d_lp, fw["entropy"], d_h)
    e_lse, e_h, _ = logp_bounds(z, fw)
    d = (e_lse + U * np.abs(fw["lse"] + offset))[:, None]
    logp = z - fw["lse"][:, None]
    p, a = np.exp(logp), np.abs(d_lp)[:, None]
    tol = a * p * np.expm1(d)
    if entropy:
        tol = tol + np.abs(d_h)[:, None] * p * (np.expm1(d) * np.abs(logp + fw["entropy"][:, None]) + np.exp(d) * (d + e_h[:, None]))
    # (the bound for a given lse, with p as large as it may be)
    given = logp_back_bounds(z, fw["lse"] - d[:, 0], d_lp, fw["entropy"], d_h, ref, "f32")
    near(f64(dz), ref, tol + given, "d_logits")
    # with lp alone the row adds up to d_lp (1 - sum p), sum p off by the same factor
    if not entropy:
        assert (np.abs(f64(dz).sum(1)) <= np.abs(d_lp) * np.expm1(d[:, 0]) + given.sum(1)).all()
