"""An iteration over an 8-bit base put together from the library's calls, as a program would: the weight quantized once,
drafts verified against the logits of the 8-bit linear, the same rows trained on with dropout on the adapter's input, back
to the clipped gradients; the same captured in a HIP graph whose replays draw new masks, on another stream and from two
threads; the native call path against the Python one."""
import threading

import numpy as np
import pytest

import paper_2309_00754_amd as H
from paper_2309_00754_amd import _binding as Bd
from oracle import (dequantize_ref, dropout_factor_ref, fp8_linear_backward_ref, fp8_linear_ref, quantize_ref, verify_ref)
from base8_helpers import backward_bounds, linear_bounds, rng_of, rounded
from gpu_helpers import host, say
from update_helpers import U, f64, near, put

pytestmark = pytest.mark.gpu

N, KD, K, V, R, S, P = 5, 7, 272, 1008, 8, 2.0, 0.1
M = N * (KD + 1)


class Step:
    """The buffers of one iteration, and the iteration itself."""

    def __init__(self, dev, seed=0):
        import torch
        r = np.random.default_rng(seed)
        bf, f = "bf16", "f32"
        self.h = put(r.normal(0, 1, (M, K)) * r.uniform(0.5, 2, K), f, dev)
        self.w, self.b = put(r.normal(1, 0.2, K), bf, dev), put(r.normal(0, 0.1, K), bf, dev)
        self.W, self.A = put(r.normal(0, K ** -0.5, (V, K)), bf, dev), put(r.normal(0, K ** -0.5, (R, K)), bf, dev)
        self.B = put(r.normal(0, R ** -0.5, (V, R)), bf, dev)
        self.hd = put(r.normal(0, 1, (N * KD, K)), bf, dev)  # the drafting model's rows
        self.drafts = torch.as_tensor(r.integers(0, V, (N, KD)).astype(np.int32)).to(dev)
        self.u = put(r.uniform(0, 1, (N, KD + 1)), f, dev)
        self.lens = torch.as_tensor(r.integers(0, KD + 1, N).astype(np.int32)).to(dev)
        self.adv, self.values, self.returns = (put(r.normal(0, 1, M), f, dev) for _ in range(3))
        self.rng = rng_of(seed, 0, dev)

        def out(*shape, dtype=torch.float32):
            return torch.full(shape, float("nan"), device=dev).to(dtype)

        def i32(*shape):
            return torch.zeros(shape, dtype=torch.int32, device=dev)

        def u8(*shape):
            return torch.zeros(shape, dtype=torch.uint8, device=dev)

        b16, nk, nv = torch.bfloat16, -(-K // 128), -(-V // 128)
        self.q, self.qs, self.qt, self.qts = u8(V, K), u8(nv, nk), u8(K, V), u8(nk, nv)
        self.x, self.mean, self.rstd = out(M, K, dtype=b16), out(M), out(M)
        self.xq, self.xs = u8(M, K), u8(M, nk)
        self.zt, self.zd = out(M, V), out(N * KD, V, dtype=b16)
        self.accepted, self.tokens, self.lp_old = i32(N), i32(N, KD + 1), out(N, KD + 1)
        self.targets = i32(M)
        self.xa, self.z = out(M, K, dtype=b16), out(M, V)
        self.lp, self.lse, self.entropy = out(M), out(M), out(M)
        self.losses, self.d_lp, self.d_v, self.dz = out(3), out(M), out(M), out(M, V, dtype=b16)
        self.dx, self.dA, self.dB = out(M, K), out(R, K), out(V, R)
        self.dh, self.flat = out(M, K), out(R * K + V * R)
        self.outs = [t.view(g.shape) for t, g in zip(self.flat.split([R * K, V * R]), (self.dA, self.dB))]
        self.norm, self.err = out(1), i32(1)

        def ws(n):
            return torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device=dev)

        self.ws_lin = ws(H.hydra_fp8_lora_linear_workspace_bytes(M, V, K, R))  # (serves the drafting rows too)
        self.ws_back = ws(H.hydra_fp8_lora_linear_backward_workspace_bytes(M, V, K, R))
        self.ws_verify = ws(H.hydra_verify_drafts_workspace_bytes(N, KD, V))

    def run(self, stream=None, own_workspaces=True):
        import torch
        st = dict(stream=stream)
        w = (lambda t: t) if own_workspaces else (lambda t: None)
        H.hydra_fp8_quantize(self.W, self.q, self.qs, 128, self.qt, self.qts, **st)
        H.hydra_layer_norm(self.h, self.w, self.b, self.x, self.mean, self.rstd, **st)
        # the rollout's logits, and the drafts
        H.hydra_fp8_lora_linear(self.x, self.q, self.qs, self.A, self.B, S, None, self.zt, workspace=w(self.ws_lin), **st)
        H.hydra_fp8_lora_linear(self.hd, self.q, self.qs, None, None, 0.0, self.zd, workspace=w(self.ws_lin), **st)
        H.hydra_verify_drafts(self.zt, self.zd, self.drafts, self.u, self.accepted, self.tokens, self.lp_old, self.lens,
                              workspace=w(self.ws_verify), err_flag=self.err, **st)
        with torch.cuda.stream(stream):
            torch.clamp(self.tokens.view(-1), min=0, out=self.targets)
        # the update, with dropout on the adapter's input
        H.hydra_dropout(self.x, self.xa, P, self.rng, **st)
        H.hydra_fp8_quantize(self.x, self.xq, self.xs, **st)
        H.hydra_fp8_lora_linear(None, self.q, self.qs, self.A, self.B, S, None, self.z, x_adapter=self.xa, xq=self.xq,
                                x_scale=self.xs, workspace=w(self.ws_lin), **st)
        H.hydra_token_logprobs(self.z, self.targets, self.lp, self.lse, self.entropy, err_flag=self.err, **st)
        H.hydra_ppo_loss(self.lp, self.lp_old.view(-1), self.adv, self.values, self.returns, N, KD + 1, self.losses, self.d_lp,
                         self.d_v, **st)
        H.hydra_token_logprobs_backward(self.z, self.targets, self.lse, self.dz, self.d_lp, err_flag=self.err, **st)
        H.hydra_fp8_lora_linear_backward(self.xa, self.qt, self.qts, self.A, self.B, S, self.dz, self.dx, self.dA, self.dB,
                                         p=P, rng=self.rng, workspace=w(self.ws_back), **st)
        H.hydra_dropout(self.dx, self.dh, P, self.rng, residual=self.h, **st)
        H.hydra_grad_clip([self.dA, self.dB], 0.05, self.norm, self.outs, **st)
        with torch.cuda.stream(stream):
            self.rng[1:].add_(1)

    NAMES = ("q", "qs", "qt", "qts", "x", "xq", "xs", "zt", "zd", "accepted", "tokens", "lp_old", "xa", "z", "lp", "lse",
             "losses", "d_lp", "dz", "dx", "dA", "dB", "dh", "norm", "flat", "err")

    def results(self):
        return {k: host(getattr(self, k).float()).copy() for k in self.NAMES}

    def clear(self, offset=0):
        for k in self.NAMES:
            t = getattr(self, k)
            t.fill_(float("nan") if t.is_floating_point() else 0)
        self.rng[1:].fill_(offset)


def test_iteration_stage_by_stage(dev):
    """Every stage against the oracle, at the inputs that the library's own earlier stages gave it."""
    import torch
    say("iteration over an 8-bit base")
    s = Step(dev)
    s.run()
    torch.cuda.synchronize()
    W = f64(s.W)
    q, e = quantize_ref(W, 128)
    Wh = dequantize_ref(q, e, 128)
    assert np.array_equal(host(s.q.view(torch.float8_e4m3fn).float()), q) and np.array_equal(host(s.qs), e + 127)
    assert torch.equal(s.qt, s.q.t()) and torch.equal(s.qts, s.qs.t())
    x, xa, hd, A, B = (f64(t) for t in (s.x, s.xa, s.hd, s.A, s.B))
    factor = dropout_factor_ref(0, 0, P, (M, K))
    near(xa, factor * x, 2.0 ** -8 * np.abs(factor * x) + 1e-38, "xa")

    def linear(x, A, B, adapter, got, y_type, which, what):
        ref = fp8_linear_ref(x, Wh, A, B, S, adapter)[which]
        tol = linear_bounds(dequantize_ref(*quantize_ref(x, 1), 1), Wh, A, B, S, y_type, adapter)[which]
        near(f64(got), ref, rounded(tol, ref, y_type), what)

    linear(x, A, B, x, s.zt, "f32", 1, "rollout's logits")
    linear(x, A, B, xa, s.z, "f32", 1, "update's logits")
    linear(hd, None, None, None, s.zd, "bf16", 0, "drafting logits")
    acc, tok, lp, odd = verify_ref(f64(s.zt).reshape(N, KD + 1, V), f64(s.zd).reshape(N, KD, V), host(s.drafts), host(s.lens),
                                   f64(s.u))
    assert np.array_equal(host(s.accepted), acc) and np.array_equal(host(s.tokens), tok) and not odd
    near(f64(s.lp_old), lp, U * np.abs(lp) + 1e-9, "lp_old")
    # the losses' gradient by torch in 64 bits, at the library's logits
    z = torch.tensor(f64(s.z), requires_grad=True)
    mine = torch.log_softmax(z, 1).gather(1, torch.tensor(host(s.targets)).long()[:, None])[:, 0]
    near(f64(s.lp), mine.detach().numpy(), 2e-5, "lp")
    # (the ratio as the library saw it: to 4e-5 of itself, and with it the gradient)
    ratio = torch.exp(mine + (torch.tensor(f64(s.lp)) - mine).detach() - torch.tensor(f64(s.lp_old).ravel()))
    adv = torch.tensor(f64(s.adv))
    (-torch.minimum(ratio * adv, ratio.clamp(0.8, 1.2) * adv).sum() / M).backward()
    dz = f64(s.dz)
    near(dz, z.grad.numpy(), (2.0 ** -8 + 2.0 ** -13) * np.abs(z.grad.numpy()) + 1e-9, "dz")
    ref = fp8_linear_backward_ref(xa, Wh, A, B, S, dz, factor)
    tol = backward_bounds(xa, Wh, A, B, S, dz, "f32", factor)
    for got, r, t, what in zip((s.dx, s.dA, s.dB), ref, (rounded(tol[0], ref[0], "f32"), tol[1], tol[2]), ("dx", "dA", "dB")):
        near(f64(got), r, t, what)
    h, dx = f64(s.h), f64(s.dx)
    near(f64(s.dh), h + factor * dx, 2 * U * (np.abs(h) + np.abs(factor * dx)) + 1e-38, "dh")
    g = np.concatenate([f64(s.dA).ravel(), f64(s.dB).ravel()])
    norm = np.sqrt((g ** 2).sum())
    near(f64(s.norm), [norm], 2 * U * norm, "norm")
    c = min(1.0, 0.05 / norm)
    near(f64(s.flat), g * c, 4 * U * np.abs(g * c) + 1e-38, "clipped")
    assert s.err.item() == 0 and host(s.rng)[1] == 1


def test_iteration_replays_in_a_hip_graph(dev):
    """Each replay draws the masks of the offset that it finds, as an eager iteration does."""
    import torch
    say("iteration in a graph")
    s, other = Step(dev, 1), Step(dev, 2)
    eager = []
    for i in range(3):
        s.run()
        torch.cuda.synchronize()
        eager.append(s.results())
    assert not np.array_equal(eager[0]["xa"], eager[1]["xa"])
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run()
    with torch.cuda.graph(g2):  # without workspaces: the capture's own memory
        s.run(own_workspaces=False)
    torch.cuda.synchronize()
    for graph in (g, g2, g):
        s.clear()
        for i in range(3):
            other.run()  # eager work between the replays
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for k, v in s.results().items():
                assert np.array_equal(v, eager[i][k]), f"replay {i}: {k}"


def test_iteration_on_another_stream(dev):
    import torch
    say("iteration on another stream")
    s = Step(dev, 3)
    s.run()
    torch.cuda.synchronize()
    want = s.results()
    side = torch.cuda.Stream(dev)
    for own in (True, False):
        s.clear()
        side.wait_stream(torch.cuda.current_stream())
        s.run(stream=side, own_workspaces=own)
        side.synchronize()
        for k, v in s.results().items():
            assert np.array_equal(v, want[k]), k


def test_two_threads_on_two_streams(dev):
    import torch
    say("two threads")
    steps = [Step(dev, 4), Step(dev, 5)]
    for s in steps:
        s.run()
    torch.cuda.synchronize()
    want = [s.results() for s in steps]
    fail = []

    def work(i):
        try:
            st = torch.cuda.Stream(dev)
            for _ in range(5):
                with torch.cuda.stream(st):
                    steps[i].rng[1:].fill_(0)
                steps[i].run(stream=st)
            st.synchronize()
        except Exception as e:  # noqa: BLE001
            fail.append(e)

    for s in steps:
        s.clear()
    torch.cuda.synchronize()
    ts = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in ts:
        t.start()
    for t in ts:
        t.join()
    assert not fail, fail
    for s, w in zip(steps, want):
        for k, v in s.results().items():
            assert np.array_equal(v, w[k]), k


def test_python_path_has_the_bits_of_the_native_one(dev, monkeypatch):
    import torch
    say("python path")
    assert not isinstance(Bd._native(), Bd._NoNative)
    s = Step(dev, 6)
    s.run()
    torch.cuda.synchronize()
    want = s.results()
    monkeypatch.setattr(Bd, "_nat", Bd._NoNative())
    for own in (True, False):
        s.clear()
        s.run(own_workspaces=own)
        torch.cuda.synchronize()
        for k, v in s.results().items():
            assert np.array_equal(v, want[k]), k
