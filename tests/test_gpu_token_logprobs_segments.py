"""Rows of logits around the length that one workgroup takes (57344): a single full one, two segments (which only rows
longer than that and no longer than the 24 KB rule asks for, or many rows, have), three, and the join over many rows."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from gpu_helpers import say
from test_gpu_token_logprobs import INF, LOW, _check
from update_helpers import TYPES, empty, f64, put

pytestmark = pytest.mark.gpu


def _sorts(V, seed):
    """A row of each sort; the largest on either side of where two segments meet, and just at it."""
    r = np.random.default_rng(seed)
    z = r.normal(0, 2, (14, V))
    half = (V // 2 + 7) // 8 * 8
    z[1], z[2], z[3] = 0.0, np.sort(z[2]), -np.sort(z[3])
    z[4, half:], z[5, :half], z[6, :] = -INF, -INF, -INF
    z[7, :] = LOW
    z[8, :], z[8, half - 1], z[8, half] = LOW, 1.0, 1.0
    z[9, V - 1], z[10, half] = np.nan, INF
    z[11] = np.round(z[11])
    z[12] += 4.0e6
    z[13, half - 20:half + 20] = 9.0
    return z, list(r.integers(0, V, 13)) + [V]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("V,top,copies", [(57344, 32, 7), (57345, 32, 7), (57345, 0, 7), (60001, 8, 7), (60001, 32, 7),
                                          (65536, 20, 7), (114688, 32, 7), (114689, 32, 7), (60001, 32, 90)])
def test_many_rows_of_one_two_and_three_segments(V, top, copies, shift, kind, dev):
    """Each sort against the oracle, its repetitions to the bit."""
    import torch
    say("segments", V, top, copies, shift, kind)
    z, tokens = _sorts(V, V + top)
    zt = put(z, kind, dev, shift, (V + 15) // 8 * 8)
    many = torch.full((copies * 14, zt.stride(0)), float("nan"), dtype=zt.dtype, device=dev)
    wide = torch.empty(many.numel() + 8, dtype=zt.dtype, device=dev)[shift:shift + many.numel()].view(many.shape)
    wide.copy_(many)
    wide.view(copies, 14, -1)[:, :, :V] = zt
    M = copies * 14
    o = {k: empty(M, "f32", dev) for k in ("lp", "lse", "entropy")}
    o["ids"] = torch.full((M, top), -7, dtype=torch.int32, device=dev) if top else None
    o["top_lp"] = empty((M, top), "f32", dev) if top else None
    o["err"] = torch.zeros(1, dtype=torch.int32, device=dev)
    H.hydra_token_logprobs(wide[:, :V], torch.tensor(tokens * copies, dtype=torch.int32, device=dev), o["lp"], o["lse"],
                           o["entropy"], o["ids"], o["top_lp"], None, o["err"])
    for k, v in o.items():
        if v is not None and k != "err":
            bits = v.view(torch.int32).view(copies, 14, -1)
            assert (bits == bits[:1]).all(), k
            o[k] = v[:14]
    _check(f64(zt), tokens, top, o, err=1)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V", [57344, 57345, 60001, 65535, 65536, 65537])
def test_single_rows(V, kind, dev):
    """One row at a time: with bf16 two segments from 57345 to 65536 logits on."""
    import torch
    say("single rows", V, kind)
    z, tokens = _sorts(V, V)
    zt = put(z, kind, dev)
    for m in (0, 2, 4, 5, 8, 11, 13):
        o = {k: empty(1, "f32", dev) for k in ("lp", "lse", "entropy")}
        o["ids"], o["top_lp"] = torch.full((1, 32), -7, dtype=torch.int32, device=dev), empty((1, 32), "f32", dev)
        o["err"] = torch.zeros(1, dtype=torch.int32, device=dev)
        tok = min(tokens[m], V - 1)
        H.hydra_token_logprobs(zt[m:m + 1], torch.tensor([tok], dtype=torch.int32, device=dev), o["lp"], o["lse"],
                               o["entropy"], o["ids"], o["top_lp"], None, o["err"])
        _check(f64(zt[m:m + 1]), [tok], 32, o)
