"""hydra_fp8_lora_linear and its backward against the oracle, within bounds derived from the arithmetic: rows from one to
several tiles, odd sizes, ranks, types, the adapter's own input, inputs already quantized, dropout's mask, values that are
not finite, repeated calls, graphs, and what lies past the last row."""
import numpy as np
import pytest

import paper_2309_00754_amd as H
from oracle import dequantize_ref, dropout_factor_ref, fp8_linear_backward_ref, fp8_linear_ref, quantize_ref
from gpu_helpers import say
from base8_helpers import (backward_bounds, f64, linear_bounds, put, quantized, rng_of, rounded)
from update_helpers import dtype, empty, near

pytestmark = pytest.mark.gpu

S = 1.5


class Linear:
    def __init__(self, seed, M, N, K, r, dev, shift=0):
        rng = np.random.default_rng(seed)
        self.M, self.N, self.K, self.r, self.dev = M, N, K, r, dev
        self.x = put(rng.normal(0, 1, (M, K)) * np.exp(rng.normal(0, 1, K)), "bf16", dev)
        self.xa = put(rng.normal(0, 1, (M, K)), "bf16", dev)
        (self.q, self.s, self.qt, self.st), self.W = quantized(f64(put(rng.normal(0, 0.02, (N, K)), "bf16", dev)), dev)
        self.A = put(rng.normal(0, K ** -0.5, (r, K)), "bf16", dev) if r else None
        self.B = put(rng.normal(0, 0.3, (N, r)), "bf16", dev, shift=shift) if r else None
        self.dy = put(rng.normal(0, 1e-3, (M, N)) * np.exp(rng.normal(0, 1, N)), "bf16", dev)

    def ab(self):
        return (None, None) if self.r == 0 else (f64(self.A), f64(self.B))

    def forward(self, y_type, xa=None, off=True, on=True, **kw):
        y = [empty((self.M, self.N), y_type, self.dev) if w else None for w in (off, on)]
        H.hydra_fp8_lora_linear(self.x, self.q, self.s, self.A, self.B, S, *y, x_adapter=xa, **kw)
        return y

    def check(self, y, y_type, xa=None, what=""):
        import torch
        torch.cuda.synchronize()
        A, B = self.ab()
        x = f64(self.x)
        a = x if xa is None else f64(xa)
        ref = fp8_linear_ref(x, self.W, A, B, S, a)
        tol = linear_bounds(dequantize_ref(*quantize_ref(x, 1), 1), self.W, A, B, S, y_type, a)
        for g, e, t, name in zip(y, ref, tol, ("y_off", "y_on")):
            if g is not None:
                near(f64(g), e, rounded(t, e, y_type), f"{what} {name}")


SIZES = [(1, 16, 16, 1), (1, 48, 160, 16), (2, 100, 272, 8), (7, 33, 1040, 5), (8, 512, 2048, 16), (16, 130, 4096, 128),
         (16, 64, 112, 64), (17, 64, 128, 16), (31, 97, 400, 3), (33, 256, 144, 32), (64, 300, 1024, 16), (65, 129, 640, 128),
         (127, 512, 528, 16), (200, 1000, 256, 64), (333, 260, 2064, 16), (130, 8200, 128, 8), (520, 3300, 144, 16),
         (1100, 2052, 272, 20), (2100, 2600, 128, 16), (40, 36, 64, 0), (5, 20, 48, 0), (230, 300, 400, 100), (401, 130, 272, 41),
        (2050, 72, 64, 128)]


@pytest.mark.parametrize("M,N,K,r", SIZES)
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
def test_linear(dev, M, N, K, r, y_type):
    say("fp8_lora_linear", M, N, K, r, y_type)
    c = Linear(M * 31 + N, M, N, K, r, dev)
    c.check(c.forward(y_type), y_type)


# Few rows and a long K, which is taken in parts; and 16384 and more outputs of few rows.
LONG = [(17, 300, 8192, 16), (40, 1030, 4112, 8), (30, 35, 32768, 64), (64, 514, 8208, 0), (100, 2050, 8192, 16),
        (33, 4100, 4096, 20), (300, 40, 16000, 128), (9, 16500, 64, 16), (5, 16389, 1040, 3), (16, 16400, 16, 0)]


@pytest.mark.parametrize("M,N,K,r", LONG)
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
def test_linear_in_parts(dev, M, N, K, r, y_type):
    import torch
    say("fp8_lora_linear", M, N, K, r, y_type)
    c = Linear(M * 7 + N, M, N, K, r, dev, shift=1)
    n = H.hydra_fp8_lora_linear_workspace_bytes(M, N, K, r)
    y = c.forward(y_type, workspace=torch.full((n,), 0xFF, dtype=torch.uint8, device=dev))
    c.check(y, y_type)
    alone = c.forward(y_type, off=False)  # (and again, from another workspace)
    assert np.array_equal(f64(alone[1]), f64(y[1]))


@pytest.mark.parametrize("M,N,K", [(112, 4100, 6000), (653, 1966, 8192)])
def test_tiles_of_128_rows_in_parts(dev, M, N, K):
    c = Linear(0, M, N, K, 16, dev)
    for y_type in ("f32", "bf16"):
        c.check(c.forward(y_type), y_type)


@pytest.mark.parametrize("M", [4, 40, 300])
def test_one_output_and_another_input_for_the_adapter(dev, M):
    c = Linear(M, M, 200, 384, 12, dev, shift=1)  # (B at an odd multiple of two bytes)
    for y_type in ("f32", "bf16"):
        both = c.forward(y_type, xa=c.xa)
        c.check(both, y_type, c.xa)
        for off, on in ((True, False), (False, True)):
            one = c.forward(y_type, xa=c.xa, off=off, on=on)
            i = 0 if off else 1
            assert np.array_equal(f64(one[i]), f64(both[i]))


@pytest.mark.parametrize("M", [3, 16, 40, 300])
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
def test_inputs_already_quantized(dev, M, y_type):
    """The bits of the call that quantizes; x itself is not needed then, but by the adapter."""
    import torch
    c = Linear(M + 1, M, 144, 400, 8, dev)
    ref = c.forward(y_type)
    xq = torch.empty((M, 400), dtype=torch.float8_e4m3fn, device=dev)
    xs = torch.empty((M, 4), dtype=torch.uint8, device=dev)
    H.hydra_fp8_quantize(c.x, xq, xs)
    for x, xa in ((c.x, None), (None, c.x)):
        y = [empty((M, 144), y_type, dev) for _ in range(2)]
        H.hydra_fp8_lora_linear(x, c.q, c.s, c.A, c.B, S, *y, x_adapter=xa, xq=xq, x_scale=xs)
        for g, e in zip(y, ref):
            assert np.array_equal(f64(g), f64(e))
    y = empty((M, 144), y_type, dev)
    H.hydra_fp8_lora_linear(None, c.q, c.s, None, None, 0.0, y, xq=xq, x_scale=xs)
    assert np.array_equal(f64(y), f64(ref[0]))


@pytest.mark.parametrize("M", [5, 16, 50, 400])
def test_repeated_calls_and_old_workspaces(dev, M):
    import torch
    c = Linear(M + 2, M, 520, 528, 16, dev)
    n = H.hydra_fp8_lora_linear_workspace_bytes(M, 520, 528, 16)
    first = c.forward("f32", workspace=torch.zeros(n, dtype=torch.uint8, device=dev))
    again = c.forward("f32", workspace=torch.full((n,), 0xFF, dtype=torch.uint8, device=dev))
    for a, b in zip(first, again):
        assert np.array_equal(f64(a), f64(b))


@pytest.mark.parametrize("M,N", [(3, 70), (20, 70), (130, 300)])
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])
def test_nothing_is_written_past_the_rows(dev, M, N, y_type, shift):
    import torch
    c = Linear(9, M, N, 160, 4, dev)
    flat = torch.full((2, shift + M * N + 300), 7.0, dtype=dtype(y_type), device=dev)
    y = [f[shift:shift + M * N].view(M, N) for f in flat]
    H.hydra_fp8_lora_linear(c.x, c.q, c.s, c.A, c.B, S, *y)
    c.check(y, y_type)
    assert (flat[:, :shift] == 7).all() and (flat[:, shift + M * N:] == 7).all()


@pytest.mark.parametrize("M", [3, 30, 200])
@pytest.mark.parametrize("y_type", ["f32", "bf16"])
def test_values_that_are_not_finite(dev, M, y_type):
    """A NaN or an infinity in x makes its row NaN, one in W its column; no other output notices."""
    import torch
    c = Linear(4, M, 80, 320, 8, dev)
    x = f64(c.x)
    x[1, 7], x[2, 300] = np.nan, np.inf
    c.x = put(x, "bf16", dev)
    c.q.view(torch.uint8)[11, 33] = 0x7F
    y = c.forward(y_type, xa=c.xa)
    torch.cuda.synchronize()
    bad = np.zeros((M, 80), bool)
    bad[1:3], bad[:, 11] = True, True
    c.W[11, 33] = 0.0
    x[1, 7], x[2, 300] = 0.0, 0.0
    for g in y:
        assert np.array_equal(np.isnan(f64(g)), bad)


@pytest.mark.parametrize("M", [3, 200])
def test_zero_rows_and_extreme_scales(dev, M):
    import torch
    c = Linear(6, M, 64, 256, 4, dev)
    x = f64(c.x)
    x[0] = 0
    x[1] *= 2.0 ** -100
    x[2] *= 2.0 ** 60
    c.x = put(x, "bf16", dev)
    for y_type in ("f32", "bf16"):
        y = c.forward(y_type, xa=c.xa)
        c.check(y, y_type, c.xa, "scales")
    y = c.forward("f32", on=False)
    assert np.all(f64(y[0])[0] == 0)


def test_update_of_nothing_is_exact(dev):
    """B = 0: y_on has the bits of y_off."""
    for M in (4, 300):
        c = Linear(8, M, 128, 256, 16, dev)
        c.B.zero_()
        for t in ("f32", "bf16"):
            y = c.forward(t)
            assert np.array_equal(f64(y[0]), f64(y[1]))


BACK = [(1, 16, 16, 1), (3, 64, 48, 8), (16, 160, 272, 128), (17, 128, 64, 16), (40, 144, 400, 5), (130, 528, 256, 64),
        (333, 272, 640, 16), (1030, 256, 2064, 16), (70, 64, 96, 0),
        (40, 8192, 304, 8), (3, 8192, 256, 16), (64, 4112, 144, 128), (1100, 144, 2608, 16), (2100, 64, 2608, 8),
        (600, 48, 3312, 20), (2100, 64, 2608, 0)]


@pytest.mark.parametrize("M,N,K,r", BACK)
@pytest.mark.parametrize("dx_type", ["f32", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.25])
def test_backward(dev, M, N, K, r, dx_type, p):
    import torch
    say("fp8_lora_linear_backward", M, N, K, r, dx_type, p)
    c = Linear(M + N, M, N, K, r, dev)
    A, B = c.ab() if r else (np.zeros((0, K)), np.zeros((N, 0)))
    factor = dropout_factor_ref(77, 5, p, (M, K)) if M * K <= 70000 else None
    if factor is None:  # (the generator is pinned element by element elsewhere)
        y = torch.empty((M, K), device=dev)
        H.hydra_dropout(torch.ones((M, K), device=dev), y, p, rng_of(77, 5, dev))
        factor = f64(y)
    dx = empty((M, K), dx_type, dev)
    dA, dB = (empty((r, K), "f32", dev), empty((N, r), "f32", dev)) if r else (None, None)
    H.hydra_fp8_lora_linear_backward(c.xa, c.qt, c.st, c.A, c.B, S, c.dy, dx, dA, dB, p=p, rng=rng_of(77, 5, dev))
    torch.cuda.synchronize()
    xa, dy = f64(c.xa), f64(c.dy)
    ref = fp8_linear_backward_ref(xa, c.W, A, B, S, dy, factor)
    tol = backward_bounds(xa, c.W, A, B, S, dy, dx_type, factor)
    near(f64(dx), ref[0], rounded(tol[0], ref[0], dx_type), "dx")
    if r:
        near(f64(dA), ref[1], tol[1], "dA")
        near(f64(dB), ref[2], tol[2], "dB")


def test_backward_outputs_one_by_one(dev):
    import torch
    c = Linear(5, 50, 96, 160, 8, dev)
    full = [empty((50, 160), "f32", dev), empty((8, 160), "f32", dev), empty((96, 8), "f32", dev)]
    rng = rng_of(1, 2, dev)
    H.hydra_fp8_lora_linear_backward(c.xa, c.qt, c.st, c.A, c.B, S, c.dy, *full, p=0.1, rng=rng)
    for i in range(3):
        o = [torch.full_like(t, float("nan")) if j == i else None for j, t in enumerate(full)]
        W = (c.qt, c.st) if i == 0 else (None, None)
        H.hydra_fp8_lora_linear_backward(c.xa if i else None, *W, c.A, c.B, S, c.dy, *o, p=0.1, rng=rng)
        assert np.array_equal(f64(o[i]), f64(full[i]))


def test_gradient_by_differences(dev):
    """dA and dB against differences of the forward's y_on (linear in each, so that a difference over a wide step is exact
    but for the forward's own bounds)."""
    import torch
    c = Linear(3, 24, 32, 64, 4, dev)
    dA, dB = empty((4, 64), "f32", dev), empty((32, 4), "f32", dev)
    H.hydra_fp8_lora_linear_backward(c.xa, None, None, c.A, c.B, S, c.dy, None, dA, dB)
    dy, xa = f64(c.dy), f64(c.xa)
    A, B = c.ab()
    tol_y = linear_bounds(dequantize_ref(*quantize_ref(f64(c.x), 1), 1), c.W, np.abs(A) + 1, np.abs(B) + 1, S, "f32", xa)[1]
    slack = 2 * (np.abs(dy) * (tol_y + 2.0 ** -24 * 50)).sum()
    for t, g in ((c.A, dA), (c.B, dB)):
        for i in [(0, 0), (3, 2), (t.shape[0] - 1, t.shape[1] - 1)]:
            keep = t[i].clone()
            y = []
            for h in (0.5, -0.5):
                t[i] = keep + h
                y.append((f64(t[i]), f64(c.forward("f32", xa=c.xa, off=False)[1])))
            t[i] = keep
            diff = (dy * (y[0][1] - y[1][1])).sum() / (y[0][0] - y[1][0])
            assert abs(diff - f64(g[i])) <= slack, (i, diff, f64(g[i]))


@pytest.mark.parametrize("M", [4, 200])
def test_a_replayed_graph_on_new_inputs(dev, M):
    import torch
    c = Linear(1, M, 256, 512, 16, dev)
    y = [empty((M, 256), "bf16", dev) for _ in range(2)]
    dx, dA, dB = empty((M, 512), "f32", dev), empty((16, 512), "f32", dev), empty((256, 16), "f32", dev)
    rng = rng_of(3, 1, dev)
    ws = torch.empty(max(H.hydra_fp8_lora_linear_workspace_bytes(M, 256, 512, 16),
                         H.hydra_fp8_lora_linear_backward_workspace_bytes(M, 256, 512, 16)), dtype=torch.uint8, device=dev)

    def step():
        H.hydra_fp8_lora_linear(c.x, c.q, c.s, c.A, c.B, S, *y, x_adapter=c.xa, workspace=ws)
        H.hydra_fp8_lora_linear_backward(c.xa, c.qt, c.st, c.A, c.B, S, c.dy, dx, dA, dB, p=0.1, rng=rng, workspace=ws)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for seed in range(3):
        r = np.random.default_rng(seed)
        for t in (c.x, c.xa, c.dy):
            t.copy_(put(r.normal(0, 1, tuple(t.shape)), "bf16", dev))
        g.replay()
        torch.cuda.synchronize()
        got = [f64(t) for t in (*y, dx, dA, dB)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (*y, dx, dA, dB)):
            assert np.array_equal(a, f64(b))
        c.check(y, "bf16", c.xa)


def test_streams_of_their_own(dev):
    import torch
    cs = [Linear(i, m, 300, 512, 16, dev) for i, m in enumerate((8, 100))]
    ss = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    ys = [c.forward("f32", stream=s) for _ in range(3) for c, s in zip(cs, ss)]
    torch.cuda.synchronize()
    for i, y in enumerate(ys):
        cs[i % 2].check(y, "f32")


def test_tensors_that_do_not_fit_are_refused(dev):
    import torch
    c = Linear(2, 4, 32, 64, 4, dev)
    y = torch.empty((4, 32), device=dev)
    with pytest.raises(TypeError):
        H.hydra_fp8_lora_linear(c.x.float(), c.q, c.s, c.A, c.B, S, y)
    with pytest.raises(TypeError):
        H.hydra_fp8_lora_linear(c.x, c.q.float(), c.s, c.A, c.B, S, y)
    with pytest.raises(ValueError):
        H.hydra_fp8_lora_linear(c.x, c.q, c.s.view(-1), c.A, c.B, S, y)
    with pytest.raises(TypeError):
        H.hydra_fp8_lora_linear(c.x, c.q, c.s, c.A, c.B, S, y, y.bfloat16())
    with pytest.raises(ValueError):
        H.hydra_fp8_lora_linear(c.x[:, :48], c.q, c.s, c.A, c.B, S, y)
    with pytest.raises(H.HydraError):
        H.hydra_fp8_lora_linear(c.x, c.q, c.s, c.A, c.B, S, y, workspace=torch.empty(16, dtype=torch.uint8, device=dev))
