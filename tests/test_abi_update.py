"""Refusals of the update step's further operators through the C ABI, without a GPU: every call below fails validation
on the host before any HIP call."""
import ctypes
import os

import pytest

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
    (dict(x=None), NULL), (dict(y=None), NULL),
    (dict(xt=2), UNSUP), (dict(wt=-1), UNSUP), (dict(yt=7), UNSUP),
    (dict(M=0), SHAPE), (dict(M=(1 << 20) + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=(1 << 21) + 1), SHAPE),
    (dict(eps=0.0), SHAPE), (dict(eps=-1e-5), SHAPE), (dict(eps=NAN), SHAPE), (dict(eps=INF), SHAPE),
    (dict(y=at(0), yt=F), SHAPE),             # over x in another type
    (dict(y=at(1)), SHAPE), (dict(mean=at(3)), SHAPE), (dict(rstd=at(4)), SHAPE), (dict(mean=at(0)), SHAPE),
    (dict(x=at(0) + 1), ALIGN), (dict(y=at(3) + 2, yt=F), ALIGN), (dict(w=at(1) + 2, wt=F), ALIGN),
    (dict(b=at(2) + 1), ALIGN), (dict(mean=at(4) + 2), ALIGN), (dict(rstd=at(5) + 1), ALIGN),
])
def test_layer_norm_rejects(kw, code):
    a = dict(x=at(0), xt=BF, w=at(1), b=at(2), wt=BF, eps=1e-5, M=4, K=64, y=at(3), yt=BF, mean=at(4), rstd=at(5))
    a.update(kw)
    assert H.lib().hydra_layer_norm(a["x"], a["xt"], a["w"], a["b"], a["wt"], a["eps"], a["M"], a["K"], a["y"], a["yt"],
                                    a["mean"], a["rstd"], None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(dy=None), NULL), (dict(x=None), NULL), (dict(mean=None), NULL), (dict(rstd=None), NULL), (dict(ws=None), NULL),
    (dict(dx=None, dw=None, db=None), NULL),
    (dict(dyt=3), UNSUP), (dict(xt=-2), UNSUP), (dict(wt=2), UNSUP), (dict(dxt=2), UNSUP),
    (dict(M=0), SHAPE), (dict(M=(1 << 20) + 1), SHAPE), (dict(K=0), SHAPE), (dict(K=(1 << 21) + 1), SHAPE),
    (dict(dx=at(0), dxt=F), SHAPE), (dict(dx=at(1), dxt=F), SHAPE), (dict(dx=at(2)), SHAPE), (dict(dw=at(5)), SHAPE),
    (dict(dw=at(7)), SHAPE), (dict(db=at(3)), SHAPE), (dict(dx=at(0), dw=at(0)), SHAPE),
    (dict(dy=at(0) + 1), ALIGN), (dict(x=at(1) + 2, xt=F), ALIGN), (dict(mean=at(3) + 2), ALIGN),
    (dict(dx=at(5) + 2, dxt=F), ALIGN), (dict(dw=at(6) + 2), ALIGN), (dict(ws=at(9) + 8), ALIGN),
    (dict(nbytes=-1), WS),
])
def test_layer_norm_backward_rejects(kw, code):
    a = dict(dy=at(0), dyt=BF, x=at(1), xt=BF, w=at(2), wt=BF, mean=at(3), rstd=at(4), M=4, K=64, dx=at(5), dxt=BF,
             dw=at(6), db=at(7), ws=at(9), nbytes=0)
    a.update(kw)
    n = H.hydra_layer_norm_backward_workspace_bytes(4, 64) + a["nbytes"]
    assert H.lib().hydra_layer_norm_backward(a["dy"], a["dyt"], a["x"], a["xt"], a["w"], a["wt"], a["mean"], a["rstd"],
                                             a["M"], a["K"], a["dx"], a["dxt"], a["dw"], a["db"], a["ws"], n, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(z=None), NULL), (dict(tok=None), NULL), (dict(lp=None), NULL),
    (dict(tok=None, lp=None, lse=None, ent=None, top=0, ids=None, tlp=None), NULL),
    (dict(ids=None), NULL), (dict(ids=None, tlp=None), NULL), (dict(top=0), NULL), (dict(top=0, ids=None), NULL),
    (dict(zt=2), UNSUP), (dict(M=0), SHAPE), (dict(M=(1 << 20) + 1), SHAPE), (dict(V=0), SHAPE),
    (dict(V=(1 << 21) + 1, ld=1 << 22), SHAPE), (dict(M=1 << 18, V=(1 << 20) + 1, ld=1 << 21), SHAPE), (dict(ld=99), SHAPE), (dict(ld=1 << 31), SHAPE),
    (dict(top=33), SHAPE), (dict(top=-1), SHAPE), (dict(V=7, top=8), SHAPE),
    (dict(lp=at(0)), SHAPE), (dict(lse=at(1)), SHAPE), (dict(ent=at(3)), SHAPE), (dict(tlp=at(5)), SHAPE),
    (dict(err=at(2)), SHAPE),
    (dict(z=at(0) + 2), ALIGN), (dict(zt=BF, z=at(0) + 1), ALIGN), (dict(tok=at(1) + 2), ALIGN),
    (dict(ids=at(5) + 2), ALIGN), (dict(err=at(7) + 1), ALIGN),
])
def test_token_logprobs_rejects(kw, code):
    a = dict(z=at(0), zt=F, ld=100, tok=at(1), M=4, V=100, top=8, lp=at(2), lse=at(3), ent=at(4), ids=at(5), tlp=at(6),
             err=at(7))
    a.update(kw)
    assert H.lib().hydra_token_logprobs(a["z"], a["zt"], a["ld"], a["tok"], a["M"], a["V"], a["top"], a["lp"], a["lse"],
                                        a["ent"], a["ids"], a["tlp"], at(9), 1 << 30, a["err"], None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(z=None), NULL), (dict(lse=None), NULL), (dict(dz=None), NULL), (dict(tok=None), NULL), (dict(ent=None), NULL),
    (dict(dlp=None, dh=None), NULL),
    (dict(zt=2), UNSUP), (dict(dt=-1), UNSUP), (dict(M=0), SHAPE), (dict(M=(1 << 20) + 1), SHAPE), (dict(V=0), SHAPE),
    (dict(V=(1 << 21) + 1, ld=1 << 22, ldd=1 << 22), SHAPE), (dict(M=1 << 20, V=1 << 19, ld=1 << 21, ldd=1 << 21), SHAPE), (dict(ld=99), SHAPE), (dict(ldd=99), SHAPE),
    (dict(ldd=1 << 31), SHAPE),
    (dict(dz=at(0), dt=BF), SHAPE), (dict(dz=at(0), ldd=104), SHAPE), (dict(dz=at(2)), SHAPE), (dict(err=at(5)), SHAPE),
    (dict(dz=at(0), err=at(0)), SHAPE),
    (dict(z=at(0) + 2), ALIGN), (dict(dz=at(6) + 2), ALIGN), (dict(dt=BF, dz=at(6) + 1), ALIGN),
    (dict(lse=at(2) + 2), ALIGN), (dict(dlp=at(4) + 2), ALIGN),
])
def test_token_logprobs_backward_rejects(kw, code):
    a = dict(z=at(0), zt=F, ld=100, tok=at(1), lse=at(2), ent=at(3), dlp=at(4), dh=at(5), M=4, V=100, dz=at(6), dt=F,
             ldd=100, err=at(7))
    a.update(kw)
    assert H.lib().hydra_token_logprobs_backward(a["z"], a["zt"], a["ld"], a["tok"], a["lse"], a["ent"], a["dlp"],
                                                 a["dh"], a["M"], a["V"], a["dz"], a["dt"], a["ldd"], a["err"],
                                                 None) == code


def _ptrs(v):
    return None if v is None else (ctypes.c_void_p * len(v))(*v)


def _i32(v):
    return None if v is None else (ctypes.c_int32 * len(v))(*v)


def _grad(g=(at(0), at(1)), t=(F, BF), n=(64, 100), max_norm=1.0, norm=at(8), outs=None, ot=None, ws=at(9), nbytes=None,
          err=None, count=None, clip=True):
    nb = H.hydra_grad_norm_workspace_bytes() if nbytes is None else nbytes
    count = len(g) if count is None and g is not None else count
    numels = None if n is None else (ctypes.c_int64 * len(n))(*n)
    if not clip:
        return H.lib().hydra_grad_norm(count, _ptrs(g), _i32(t), numels, norm, ws, nb, None)
    return H.lib().hydra_grad_clip(count, _ptrs(g), _i32(t), numels, max_norm, norm, _ptrs(outs), _i32(ot), ws, nb, err,
                                   None)


@pytest.mark.parametrize("clip", [True, False])
@pytest.mark.parametrize("kw,code", [
    (dict(count=0), SHAPE), (dict(count=4097), SHAPE), (dict(g=None, count=2), NULL), (dict(t=None), NULL),
    (dict(n=None), NULL), (dict(norm=None), NULL), (dict(ws=None), NULL), (dict(g=(at(0), None)), NULL),
    (dict(t=(F, 2)), UNSUP), (dict(n=(64, -1)), SHAPE), (dict(n=((1 << 40) + 1, 1)), SHAPE),
    (dict(n=(1 << 40, 1)), SHAPE), (dict(g=(at(0) + 2, at(1))), ALIGN), (dict(g=(at(0), at(1) + 1)), ALIGN),
    (dict(norm=at(8) + 2), ALIGN), (dict(ws=at(9) + 8), ALIGN), (dict(nbytes=16), WS),
])
def test_grad_norm_rejects(clip, kw, code):
    assert _grad(clip=clip, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(max_norm=-1.0), SHAPE), (dict(max_norm=NAN), SHAPE), (dict(err=at(7) + 1), ALIGN), (dict(err=at(8)), SHAPE),
    (dict(outs=(at(2), at(3))), NULL), (dict(ot=(F, F)), NULL), (dict(outs=(at(2), None), ot=(F, F)), NULL),
    (dict(outs=(at(2), at(3)), ot=(F, 5)), UNSUP), (dict(outs=(at(2) + 2, at(3)), ot=(F, F)), ALIGN),
    # in place: the same tensor twice, two that overlap, the norm or the flag inside one
    (dict(g=(at(0), at(0)), t=(F, F)), SHAPE), (dict(g=(at(1), at(0), at(1) + 252), t=(F, F, F), n=(64, 64, 64)), SHAPE),
    (dict(norm=at(0) + 16), SHAPE), (dict(err=at(1) + 100), SHAPE),
    # out of place: one out twice, outs that overlap in any order, an out over another gradient, over its own in
    # another type or shifted, a gradient that stands twice and is written once
    (dict(outs=(at(2), at(2)), ot=(F, BF)), SHAPE), (dict(outs=(at(2) + 100, at(2)), ot=(F, F)), SHAPE),
    (dict(outs=(at(1), at(2)), ot=(F, BF)), SHAPE), (dict(outs=(at(1) + 192, at(2)), ot=(F, BF)), SHAPE),
    (dict(outs=(at(0), at(2)), ot=(BF, BF)), SHAPE), (dict(outs=(at(0) + 4, at(2)), ot=(F, BF)), SHAPE),
    (dict(g=(at(0), at(0)), t=(F, F), n=(64, 64), outs=(at(0), at(2)), ot=(F, F)), SHAPE),
    (dict(outs=(at(2), at(3)), ot=(F, F), norm=at(3) + 8), SHAPE),
])
def test_grad_clip_rejects(kw, code):
    assert _grad(**kw) == code


def test_workspace_sizes():
    b = ctypes.c_size_t(0)
    L = H.lib()
    assert L.hydra_layer_norm_backward_workspace_bytes(0, 8, ctypes.byref(b)) == SHAPE
    assert L.hydra_layer_norm_backward_workspace_bytes(8, (1 << 21) + 1, ctypes.byref(b)) == SHAPE
    assert L.hydra_layer_norm_backward_workspace_bytes(8, 8, None) == NULL
    assert L.hydra_token_logprobs_workspace_bytes(8, 7, 8, ctypes.byref(b)) == SHAPE
    assert L.hydra_token_logprobs_workspace_bytes(1 << 20, 1 << 19, 8, ctypes.byref(b)) == SHAPE
    assert L.hydra_token_logprobs_workspace_bytes(8, 100, 33, ctypes.byref(b)) == SHAPE
    assert L.hydra_token_logprobs_workspace_bytes(8, 100, 8, None) == NULL
    assert L.hydra_grad_norm_workspace_bytes(None) == NULL
    # every size that a call accepts has a workspace that fits the card many times over at sizes in use
    for M, K in ((1, 1), (4096, 2048), (1 << 20, 4096), (16, 1 << 21)):
        assert 0 < H.hydra_layer_norm_backward_workspace_bytes(M, K) < 1 << 29
    for M, V, k in ((1, 1, 0), (6, 50272, 8), (4096, 50272, 32), (1, 1 << 21, 32)):
        assert 0 <= H.hydra_token_logprobs_workspace_bytes(M, V, k) < 1 << 28
