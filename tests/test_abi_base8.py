"""Refusals of the 8-bit base's operators, dropout and draft verification through the C ABI, without a GPU: every call
below fails validation on the host before any HIP call."""
import ctypes
import os

import pytest
import torch

import paper_2309_00754_amd as H

pytestmark = pytest.mark.skipif(not os.path.exists(H.LIB_PATH), reason="libhydra.so not built")

P = 0x100000  # fake device addresses, never dereferenced
BF, F = H.HYDRA_BF16, H.HYDRA_F32
NULL, SHAPE, ALIGN, UNSUP, WS = (H.HYDRA_ERR_NULL, H.HYDRA_ERR_SHAPE, H.HYDRA_ERR_ALIGN, H.HYDRA_ERR_UNSUPPORTED,
                                 H.HYDRA_ERR_WORKSPACE)
INF, NAN = float("inf"), float("nan")


def at(i):
    return P + 0x10000 * i


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(q=None), NULL), (dict(s=None), NULL), (dict(qt=None), NULL), (dict(st=None), NULL),
    (dict(xt=2), UNSUP), (dict(rows=64), UNSUP), (dict(rows=0), UNSUP), (dict(rows=1), UNSUP),
    (dict(M=0), SHAPE), (dict(M=(1 << 21) + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=(1 << 21) + 1), SHAPE),
    (dict(M=1 << 21, K=1 << 17), SHAPE), (dict(M=1 << 21, K=1 << 14, rows=1, qt=None, st=None), SHAPE),
    (dict(q=at(0)), SHAPE), (dict(qt=at(1)), SHAPE), (dict(s=at(3)), SHAPE),
    (dict(x=at(0) + 1), ALIGN), (dict(x=at(0) + 2, xt=F), ALIGN),
])
def test_quantize_rejects(kw, code):
    a = dict(x=at(0), xt=BF, M=130, K=60, rows=128, q=at(1), s=at(2), qt=at(3), st=at(4))
    a.update(kw)
    assert H.lib().hydra_fp8_quantize(a["x"], a["xt"], a["M"], a["K"], a["rows"], a["q"], a["s"], a["qt"], a["st"],
                                      None) == code


LIN = dict(x=at(0), xa=None, xq=None, xs=None, W=at(1), ws=at(2), A=at(3), B=at(4), M=40, N=64, K=64, r=8, off=at(5),
           on=at(6), yt=F, w=at(9), nb=1 << 30)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(W=None), NULL), (dict(ws=None), NULL), (dict(A=None), NULL), (dict(B=None), NULL),
    (dict(off=None, on=None), NULL), (dict(xq=at(7)), NULL), (dict(xs=at(7)), NULL), (dict(w=None), NULL),
    (dict(x=None, xq=at(7), xs=at(8)), NULL),  # the adapter has no input
    (dict(yt=2), UNSUP), (dict(M=0), SHAPE), (dict(M=(1 << 20) + 1), SHAPE), (dict(N=0), SHAPE),
    (dict(N=(1 << 21) + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=72), SHAPE), (dict(K=(1 << 21) + 16), SHAPE),
    (dict(r=-1), SHAPE), (dict(r=129), SHAPE), (dict(M=1 << 20, N=1 << 20), SHAPE),
    (dict(off=at(6)), SHAPE), (dict(on=at(0)), SHAPE), (dict(off=at(4)), SHAPE), (dict(on=at(7), xa=at(7)), SHAPE),
    (dict(x=at(0) + 8), ALIGN), (dict(xa=at(7) + 2), ALIGN), (dict(W=at(1) + 8), ALIGN), (dict(A=at(3) + 2), ALIGN),
    (dict(B=at(4) + 1), ALIGN), (dict(off=at(5) + 2), ALIGN), (dict(on=at(6) + 1, yt=BF, off=None), ALIGN),
    (dict(w=at(9) + 8), ALIGN), (dict(nb=-1), WS), (dict(xq=at(7) + 4, xs=at(8)), ALIGN),
])
def test_linear_rejects(kw, code):
    a = {**LIN, **kw}
    nb = H.hydra_fp8_lora_linear_workspace_bytes(40, 64, 64, 8) - 1 if a["nb"] < 0 else a["nb"]
    assert H.lib().hydra_fp8_lora_linear(a["x"], a["xa"], a["xq"], a["xs"], a["W"], a["ws"], a["A"], a["B"], 1.0, a["M"],
                                         a["N"], a["K"], a["r"], a["off"], a["on"], a["yt"], a["w"], nb, None) == code


BACK = dict(x=at(0), W=at(1), ws=at(2), A=at(3), B=at(4), dy=at(5), M=40, N=64, K=80, r=8, p=0.1, rng=at(6), dx=at(7),
            dxt=F, dA=at(8), dB=at(9), w=at(10), nb=1 << 30)


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), NULL), (dict(W=None), NULL), (dict(ws=None), NULL), (dict(A=None), NULL), (dict(B=None), NULL),
    (dict(x=None), NULL), (dict(rng=None), NULL), (dict(dx=None, dA=None, dB=None), NULL), (dict(r=0, dx=None), NULL),
    (dict(w=None), NULL), (dict(dxt=3), UNSUP), (dict(M=0), SHAPE), (dict(M=(1 << 20) + 1), SHAPE), (dict(N=72), SHAPE),
    (dict(K=72), SHAPE), (dict(K=0), SHAPE), (dict(r=129), SHAPE), (dict(p=-0.1), SHAPE), (dict(p=1.5), SHAPE),
    (dict(p=NAN), SHAPE), (dict(dx=at(5)), SHAPE), (dict(dA=at(3)), SHAPE), (dict(dB=at(8)), SHAPE), (dict(dx=at(6)), SHAPE),
    (dict(x=at(0) + 8), ALIGN), (dict(W=at(1) + 1), ALIGN), (dict(dy=at(5) + 2), ALIGN), (dict(rng=at(6) + 4), ALIGN),
    (dict(dx=at(7) + 2), ALIGN), (dict(dA=at(8) + 1), ALIGN), (dict(w=at(10) + 4), ALIGN), (dict(nb=-1), WS),
])
def test_linear_backward_rejects(kw, code):
    a = {**BACK, **kw}
    nb = H.hydra_fp8_lora_linear_backward_workspace_bytes(40, 64, 80, 8) - 1 if a["nb"] < 0 else a["nb"]
    assert H.lib().hydra_fp8_lora_linear_backward(
        a["x"], a["W"], a["ws"], a["A"], a["B"], 1.0, a["dy"], a["M"], a["N"], a["K"], a["r"], a["p"], a["rng"], a["dx"],
        a["dxt"], a["dA"], a["dB"], a["w"], nb, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), NULL), (dict(rng=None), NULL), (dict(y=None), NULL), (dict(xt=2), UNSUP), (dict(rt=-1), UNSUP),
    (dict(yt=5), UNSUP), (dict(n=0), SHAPE), (dict(n=(1 << 34) + 1), SHAPE), (dict(p=-1e-9), SHAPE), (dict(p=1.01), SHAPE),
    (dict(p=NAN), SHAPE), (dict(y=at(0), yt=F), SHAPE), (dict(y=at(1), yt=BF, rt=F), SHAPE), (dict(y=at(2)), SHAPE),
    (dict(x=at(0) + 1), ALIGN), (dict(r=at(1) + 2, rt=F), ALIGN), (dict(y=at(3) + 1), ALIGN), (dict(rng=at(2) + 4), ALIGN),
])
def test_dropout_rejects(kw, code):
    a = dict(x=at(0), xt=BF, r=at(1), rt=BF, p=0.1, rng=at(2), n=100, y=at(3), yt=BF)
    a.update(kw)
    assert H.lib().hydra_dropout(a["x"], a["xt"], a["r"], a["rt"], a["p"], a["rng"], a["n"], a["y"], a["yt"], None) == code


VER = dict(z=at(0), zt=F, ld=100, d=at(1), dt=F, ldd=100, drafts=at(2), lens=at(3), u=at(4), n=3, k=4, V=100, T=1.0,
           acc=at(5), tok=at(6), lp=at(7), w=at(9), nb=1 << 30, err=at(8))


@pytest.mark.parametrize("kw,code", [
    (dict(z=None), NULL), (dict(u=None), NULL), (dict(acc=None), NULL), (dict(tok=None), NULL), (dict(drafts=None), NULL),
    (dict(w=None), NULL), (dict(zt=2), UNSUP), (dict(dt=-1), UNSUP), (dict(n=0), SHAPE), (dict(k=-1), SHAPE),
    (dict(k=129), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 21) + 1, ld=1 << 22, ldd=1 << 22), SHAPE),
    (dict(n=1 << 18), SHAPE), (dict(n=1 << 14, V=1 << 20, ld=1 << 20, ldd=1 << 20), SHAPE), (dict(ld=99), SHAPE),
    (dict(ld=1 << 31), SHAPE), (dict(ldd=99), SHAPE), (dict(T=0.0), SHAPE), (dict(T=-1.0), SHAPE), (dict(T=NAN), SHAPE),
    (dict(T=INF), SHAPE), (dict(T=1e-40), SHAPE),
    (dict(acc=at(0)), SHAPE), (dict(tok=at(2)), SHAPE), (dict(lp=at(4)), SHAPE), (dict(err=at(3)), SHAPE),
    (dict(lp=at(6)), SHAPE), (dict(z=at(0) + 2), ALIGN), (dict(d=at(1) + 1, dt=BF), ALIGN), (dict(u=at(4) + 2), ALIGN),
    (dict(lens=at(3) + 1), ALIGN), (dict(tok=at(6) + 2), ALIGN), (dict(err=at(8) + 2), ALIGN), (dict(w=at(9) + 8), ALIGN),
    (dict(nb=-1), WS),
])
def test_verify_drafts_rejects(kw, code):
    a = {**VER, **kw}
    nb = H.hydra_verify_drafts_workspace_bytes(3, 4, 100) - 1 if a["nb"] < 0 else a["nb"]
    assert H.lib().hydra_verify_drafts(a["z"], a["zt"], a["ld"], a["d"], a["dt"], a["ldd"], a["drafts"], a["lens"], a["u"],
                                       a["n"], a["k"], a["V"], a["T"], a["acc"], a["tok"], a["lp"], a["w"], nb, a["err"],
                                       None) == code


def test_workspace_sizes():
    b = ctypes.c_size_t(0)
    L = H.lib()
    assert L.hydra_fp8_lora_linear_workspace_bytes(0, 64, 64, 8, ctypes.byref(b)) == SHAPE
    assert L.hydra_fp8_lora_linear_workspace_bytes(8, 64, 72, 8, ctypes.byref(b)) == SHAPE
    assert L.hydra_fp8_lora_linear_workspace_bytes(8, 64, 64, 129, ctypes.byref(b)) == SHAPE
    assert L.hydra_fp8_lora_linear_workspace_bytes(8, 64, 64, 8, None) == NULL
    assert L.hydra_fp8_lora_linear_backward_workspace_bytes(8, 64, 72, 8, ctypes.byref(b)) == SHAPE
    assert L.hydra_fp8_lora_linear_backward_workspace_bytes(8, 64, 64, 8, None) == NULL
    assert L.hydra_verify_drafts_workspace_bytes(8, 129, 64, ctypes.byref(b)) == SHAPE
    assert L.hydra_verify_drafts_workspace_bytes(8, 4, 64, None) == NULL
    for M, K, r in ((1, 16, 0), (8, 4096, 16), (2048, 11008, 128), (1 << 20, 4096, 16)):
        n = H.hydra_fp8_lora_linear_workspace_bytes(M, 4096, K, r)
        assert M * K <= n <= 2 * M * K + 40 * M * 128 + (1 << 26)
    for n, k, V in ((1, 0, 1), (64, 7, 50272), (1, 128, 1 << 21)):
        assert 0 < H.hydra_verify_drafts_workspace_bytes(n, k, V) < 1 << 24


@pytest.mark.parametrize("N,K,r", [(16, 16, 1), (4096, 4096, 16), (4096, 11008, 64), (50272, 512, 128), (130, 32768, 0)])
def test_the_largest_calls_workspace_serves_fewer_rows(N, K, r):
    got = [H.hydra_fp8_lora_linear_workspace_bytes(M, N, K, r) for M in list(range(1, 300)) + list(range(300, 20000, 97))]
    assert got == sorted(got)


def test_host_tensors_are_refused():
    x, b = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 1, dtype=torch.uint8)
    q, y = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 4)
    rng, i = torch.zeros(2, dtype=torch.int64), torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError):
        H.hydra_fp8_quantize(x, q, b)
    with pytest.raises(ValueError):
        H.hydra_fp8_quantize(x, q, b, 64)
    with pytest.raises(ValueError):
        H.hydra_fp8_lora_linear(x, q, b[:1], None, None, 1.0, y)
    with pytest.raises(ValueError):
        H.hydra_fp8_lora_linear(None, q, b[:1], None, None, 1.0, y)
    with pytest.raises(ValueError):
        H.hydra_fp8_lora_linear_backward(None, q, b[:1], None, None, 1.0, x, torch.zeros(4, 4))
    with pytest.raises(ValueError):
        H.hydra_dropout(x, x.clone(), 0.1, rng)
    with pytest.raises(ValueError):
        H.hydra_verify_drafts(torch.zeros(1, 8), None, None, torch.zeros(1, 1), i[0], i)
