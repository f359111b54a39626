"""The operators of a Hydra-PPO iteration whose frozen base is held in 8 bits, as cases to time.

A case is a dict of plain values; "kind" names the entry point it goes through:

* quantize   bf16 or fp32 rows, or a weight, to e4m3 with a power-of-two scale for each block of 128 (hydra_fp8_quantize)
* linear     the dual-output linear over the 8-bit base, LoRA update on top (hydra_fp8_lora_linear)
* backward   its gradients, with the mask of the adapter's dropout made again (hydra_fp8_lora_linear_backward)
* dropout    dropout from a counter-based generator, onto a residual or alone (hydra_dropout)
* verify     drafted tokens against the target's probabilities, the next token sampled (hydra_verify_drafts)

Sizes are those of the repository's Llama-7B and OPT-1.3b configurations (hidden 4096 and 2048, MLP 11008 and 8192,
vocabulary 32000 and 50272, ranks 16 and 128, batches of 4 and 8 sequences of 512 tokens) and ragged ones between them.
"""
import math

import torch

own = False

BF16, F32, F64, I64, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.int64, torch.float8_e4m3fn
TYPES = {"bf16": BF16, "f32": F32}
BYTES = {"bf16": 2, "f32": 4}
BLOCK = 128
WORKSPACE = 192 << 20  # bytes of scratch memory that a program keeps for whichever call comes


def listed():
    return [
        # a prefill's activations before the linears: 4 x 512 tokens of Llama-7B
        dict(name="quantize_rows", kind="quantize", M=2048, K=4096, x="bf16", block_rows=1, transposed=False),
        # a frozen MLP weight, once after loading: the copy that the forward reads and the one that the backward reads
        dict(name="quantize_weight", kind="quantize", M=11008, K=4096, x="bf16", block_rows=128, transposed=True),
        # one token for each of 4 sequences through a projection of OPT-1.3b: latency alone
        dict(name="linear_token", kind="linear", M=4, N=2048, K=2048, r=16, y="f32", off=False, on=True),
        # a step that verifies seven drafted tokens through Llama-7B's MLP: W is read once for all eight rows
        dict(name="linear_drafts", kind="linear", M=8, N=11008, K=4096, r=16, y="f32", off=False, on=True),
        # a ragged prompt through the MLP's way back
        dict(name="linear_prompt", kind="linear", M=333, N=4096, K=11008, r=16, y="f32", off=True, on=True),
        # a batch of 4 x 512 tokens, reference and actor from one product
        dict(name="linear_batch", kind="linear", M=2048, N=11008, K=4096, r=16, y="bf16", off=True, on=True),
        # the update stage over that batch, one projection, the usual adapter dropout
        dict(name="backward_batch", kind="backward", M=2048, N=4096, K=4096, r=16, p=0.05, dx="f32"),
        # one ragged sequence through OPT-1.3b's MLP at the paper's rank 128, no dropout
        dict(name="backward_sequence", kind="backward", M=250, N=8192, K=2048, r=128, p=0.0, dx="f32"),
        # the adapter's input of a batch
        dict(name="dropout_adapter", kind="dropout", M=2048, K=4096, x="bf16", res="none", y="bf16", p=0.05),
        # OPT-1.3b's residual stream: 8 x 512 tokens, the linear's fp32 output onto it
        dict(name="dropout_residual", kind="dropout", M=4096, K=2048, x="f32", res="f32", y="f32", p=0.1),
        # one sequence with five drafts: what every step of its rollout waits for
        dict(name="verify_one", kind="verify", n=1, k=5, V=32000, z="f32", zd="f32", ragged=False, temperature=1.0),
        # a rollout batch over OPT-1.3b's vocabulary, up to seven drafts each
        dict(name="verify_batch", kind="verify", n=64, k=7, V=50272, z="f32", zd="bf16", ragged=True, temperature=0.8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "linear", "backward", "backward", "dropout", "verify", "verify"])

    def t():
        return rng.choice(["bf16", "f32"])

    if kind == "quantize":
        K = rng.choice([2048, 4096, 8192, 11008, 16 * _log(rng, 1, 688), _log(rng, 1, 11008)])
        rows = rng.random() < 0.5
        M = min(_log(rng, 1, 11008), 11008 * 4096 // K)
        return dict(kind=kind, M=M, K=K, x=t(), block_rows=1 if rows else 128, transposed=not rows and rng.random() < 0.7)
    if kind == "dropout":
        K = rng.choice([2048, 4096, 11008, _log(rng, 1, 11008)])
        M = min(_log(rng, 1, 16384), (1 << 24) // K)
        return dict(kind=kind, M=M, K=K, x=t(), res=rng.choice(["none", "bf16", "f32"]), y=t(),
                    p=rng.choice([0.0, 0.05, 0.1, 0.5, rng.random()]))
    if kind == "verify":
        V = rng.choice([32000, 50272, _log(rng, 1000, 60000)])
        k = rng.choice([0, 1, 3, 5, 7, rng.randrange(16)])
        n = max(1, min(_log(rng, 1, 128), 64 * 15 * 50272 // (V * (2 * k + 1))))
        return dict(kind=kind, n=n, k=k, V=V, z=t(), zd=rng.choice(["none", "bf16", "f32"]), ragged=rng.random() < 0.5,
                    temperature=rng.choice([1.0, 0.7, 1.3]))
    N = rng.choice([2048, 4096, 8192, 11008, 16 * _log(rng, 4, 688)])
    K = rng.choice([2048, 4096, 8192, 11008, 16 * _log(rng, 4, 688)])
    r = rng.choice([8, 16, 16, 64, 128, rng.randrange(1, 129)])
    if kind == "linear":
        N = rng.choice([N, N, N, _log(rng, 64, 11008)])
        M = min(_log(rng, 1, 4096), 2048 * 11008 * 4096 // (N * K))
        off, on = rng.choice([(True, True), (False, True), (True, False)])
        return dict(kind=kind, M=M, N=N, K=K, r=r, y=t(), off=off, on=on)
    M = min(_log(rng, 1, 4096), 2048 * 4096 * 4096 // (N * K))
    return dict(kind=kind, M=M, N=N, K=K, r=r, p=rng.choice([0.0, 0.05, 0.1]), dx=t())


class _Draw:
    """Seeded tensors on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, *shape, std=1.0, mean=0.0, dtype=F32):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=F32).mul_(std).add_(mean).to(dtype)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda", dtype=F32)

    def whole(self, lo, hi, *shape, dtype=torch.int32):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=dtype)


def _up(a, b):
    return -(-a // b)


def _blocks(x, rows):
    """x with each block of `rows` x 128 values as two axes of its own, zeros past the edges: [R, rows, C, 128]."""
    M, K = x.shape
    x = torch.nn.functional.pad(x, (0, _up(K, BLOCK) * BLOCK - K, 0, _up(M, rows) * rows - M))
    return x.view(_up(M, rows), rows, _up(K, BLOCK), BLOCK)


def _spread(e, rows, M, K):
    """A value for each block as one for each element."""
    return e.repeat_interleave(rows, 0)[:M].repeat_interleave(BLOCK, 1)[:, :K]


def _power(e):
    """2^e in fp32, whole e from -127 to 127, exactly (by its bits)."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).view(F32)


def _quantize(x, rows):
    """(e4m3 values, scale bytes): the least scale 2^e, e >= -127, that brings the block's largest magnitude to 448 or less."""
    M, K = x.shape
    x = x.to(F32)
    finite = torch.isfinite(x)
    a = _blocks(torch.where(finite, x, 0.0).abs(), rows).amax((1, 3))
    f, e = torch.frexp(a)  # 448 is 0.875 * 2^9
    e = torch.where(a > 0, e - 9 + (f > 0.875), -127).clamp(min=-127).to(torch.int32)
    q = torch.where(finite, x * _spread(_power(-e), rows, M, K), math.nan)
    return q.to(E4M3), (e + 127).to(torch.uint8)


def _values(q, scale, rows):
    """What quantized rows stand for, in fp32."""
    M, K = q.shape
    return q.to(F32) * _spread(_power(scale.to(torch.int32) - 127), rows, M, K)


def _inputs(case, seed):
    d, kind, i = _Draw(seed), case["kind"], {}
    if kind in ("quantize", "dropout"):
        M, K = case["M"], case["K"]
        # hidden states with channels of their own width, a few of them far wider; a weight is narrower and even
        x = d.normal(M, K, std=0.02) if case.get("block_rows") == 128 else d.normal(M, K) * torch.exp(d.normal(K))
        i["x"] = x.to(TYPES[case["x"]])
        if kind == "dropout":
            i["res"] = None if case["res"] == "none" else d.normal(M, K, std=3.0, dtype=TYPES[case["res"]])
            i["rng"] = torch.stack([d.whole(-(1 << 62), 1 << 62, 1, dtype=I64)[0], d.whole(0, 1 << 40, 1, dtype=I64)[0]])
        return i
    if kind == "verify":
        n, k, V = case["n"], case["k"], case["V"]
        z = d.normal(n, k + 1, V, std=2.5)
        # the draft's logits: the target's, off by about one
        zd = (z[:, :k] + d.normal(n, k, V, std=0.7)).to(TYPES["f32" if case["zd"] == "none" else case["zd"]])
        noise = d.uniform(n, k, V).clamp_(1e-9, 1 - 1e-7).log_().neg_().log_().neg_()
        i["drafts"] = noise.add_(zd, alpha=1.0 / case["temperature"]).argmax(2).to(torch.int32)
        if case["zd"] == "none":  # drafts looked up in the prompt: no distribution, right more often than not
            i["drafts"] = torch.where(d.uniform(n, k) < 0.7, z[:, :k].argmax(2).to(torch.int32), i["drafts"])
            z.scatter_add_(2, z.argmax(2, keepdim=True), torch.full((n, k + 1, 1), 6.0, device="cuda"))
        i["z"] = z.to(TYPES[case["z"]]).view(n * (k + 1), V)
        i["zd"] = None if case["zd"] == "none" or k == 0 else zd.view(n * k, V)
        i["u"] = d.uniform(n, k + 1)
        i["lens"] = d.whole(0, k + 1, n) if case["ragged"] else None
        return i
    M, N, K, r = case["M"], case["N"], case["K"], case["r"]
    rows, cols = (M, K) if kind == "linear" else (M, N)  # of what is quantized in the call
    wide = torch.exp(d.normal(K, std=0.5))
    i["x"] = (d.normal(M, K) * wide).to(BF16)
    # the frozen weight, as the forward reads it [N x K] or the backward [K x N]
    w = d.normal(*((N, K) if kind == "linear" else (K, N)), std=0.02, dtype=BF16)
    i["wq"], i["ws"] = _quantize(w, BLOCK)
    i["A"] = d.normal(r, K, std=K ** -0.5, dtype=BF16)
    i["B"] = d.normal(N, r, std=0.02, dtype=BF16)
    i["s"] = 32.0 / r
    if kind == "backward":
        i["dy"] = d.normal(rows, cols, std=1e-3, dtype=BF16)
        i["rng"] = torch.stack([d.whole(-(1 << 62), 1 << 62, 1, dtype=I64)[0], d.whole(0, 1 << 40, 1, dtype=I64)[0]])
    return i


def prepare(case, seed):
    """The inputs, and the output buffers and workspace that a program allocates once."""
    s = _inputs(case, seed)
    s["case"], kind = case, case["kind"]

    def out(*shape, dtype=F32):
        return torch.empty(shape, device="cuda", dtype=dtype)

    if kind == "quantize":
        M, K, rows = case["M"], case["K"], case["block_rows"]
        s["q"], s["scale"] = out(M, K, dtype=E4M3), out(_up(M, rows), _up(K, BLOCK), dtype=torch.uint8)
        t = case["transposed"]
        s["qt"] = out(K, M, dtype=E4M3) if t else None
        s["scale_t"] = out(_up(K, BLOCK), _up(M, BLOCK), dtype=torch.uint8) if t else None
    elif kind == "linear":
        y = TYPES[case["y"]]
        s["y_off"] = out(case["M"], case["N"], dtype=y) if case["off"] else None
        s["y_on"] = out(case["M"], case["N"], dtype=y) if case["on"] else None
    elif kind == "backward":
        s["dx"] = out(case["M"], case["K"], dtype=TYPES[case["dx"]])
        s["dA"], s["dB"] = out(case["r"], case["K"]), out(case["N"], case["r"])
    elif kind == "dropout":
        s["y"] = out(case["M"], case["K"], dtype=TYPES[case["y"]])
    else:
        n, k = case["n"], case["k"]
        s["accepted"], s["tokens"] = out(n, dtype=torch.int32), out(n, k + 1, dtype=torch.int32)
        s["lp"] = out(n, k + 1)
    s["workspace"] = out(WORKSPACE, dtype=torch.uint8)
    return s


OUTPUTS = {"quantize": ("q", "scale", "qt", "scale_t"), "linear": ("y_off", "y_on"), "backward": ("dx", "dA", "dB"),
           "dropout": ("y",), "verify": ("accepted", "tokens", "lp")}


def _run_own(s):
    import paper_2309_00754_amd as H
    case, kind = s["case"], s["case"]["kind"]
    if kind == "quantize":
        H.hydra_fp8_quantize(s["x"], s["q"], s["scale"], case["block_rows"], s["qt"], s["scale_t"])
    elif kind == "linear":
        H.hydra_fp8_lora_linear(s["x"], s["wq"], s["ws"], s["A"], s["B"], s["s"], s["y_off"], s["y_on"],
                                workspace=s["workspace"])
    elif kind == "backward":
        H.hydra_fp8_lora_linear_backward(s["x"], s["wq"], s["ws"], s["A"], s["B"], s["s"], s["dy"], s["dx"], s["dA"],
                                         s["dB"], p=case["p"], rng=s["rng"], workspace=s["workspace"])
    elif kind == "dropout":
        H.hydra_dropout(s["x"], s["y"], case["p"], s["rng"], residual=s["res"])
    else:
        H.hydra_verify_drafts(s["z"], s["zd"], s["drafts"], s["u"], s["accepted"], s["tokens"], s["lp"], s["lens"],
                              temperature=case["temperature"], workspace=s["workspace"])
    return {k: s[k] for k in OUTPUTS[kind]}


def _keep(rng, p, M, K):
    """(whether an element is kept, what it is multiplied by): sixteen bits each of Philox4x32-10, eight elements to a
    counter value, in 64-bit whole numbers that hold 32 bits."""
    low = 0xFFFFFFFF
    drop = int(round(p * 65536))
    c0 = torch.arange(_up(M * K, 8), device="cuda", dtype=I64)
    c1, c2, c3 = c0 >> 32, (rng[1] & low).expand_as(c0), ((rng[1] >> 32) & low).expand_as(c0)
    c0, k0, k1 = c0 & low, rng[0] & low, (rng[0] >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], 1)
    bits = torch.stack([words & 0xFFFF, words >> 16], 2).view(-1)[:M * K].view(M, K)
    return bits >= drop, (65536.0 / (65536 - drop) if drop < 65536 else 0.0)


def run(s):
    if own:
        return _run_own(s)
    case, kind = s["case"], s["case"]["kind"]
    if kind == "quantize":
        q, scale = _quantize(s["x"], case["block_rows"])
        t = case["transposed"]
        return {"q": q, "scale": scale, "qt": q.t().contiguous() if t else None,
                "scale_t": scale.t().contiguous() if t else None}
    if kind == "linear":
        x = s["x"].to(F32)
        y = _values(*_quantize(x, 1), 1) @ _values(s["wq"], s["ws"], BLOCK).t()
        o = {"y_off": y.to(TYPES[case["y"]]) if case["off"] else None, "y_on": None}
        if case["on"]:
            o["y_on"] = (y + s["s"] * ((x @ s["A"].to(F32).t()) @ s["B"].to(F32).t())).to(TYPES[case["y"]])
        return o
    if kind == "backward":
        x, dy, A, B = (s[n].to(F32) for n in ("x", "dy", "A", "B"))
        back = s["s"] * (dy @ B)
        through = back @ A
        if case["p"] > 0:
            keep, c = _keep(s["rng"], case["p"], case["M"], case["K"])
            through = torch.where(keep, through * c, 0.0)
        dx = _values(*_quantize(dy, 1), 1) @ _values(s["wq"], s["ws"], BLOCK).t() + through
        return {"dx": dx.to(TYPES[case["dx"]]), "dA": back.t() @ x, "dB": s["s"] * (dy.t() @ (x @ A.t()))}
    if kind == "dropout":
        keep, c = _keep(s["rng"], case["p"], case["M"], case["K"])
        y = torch.where(keep, s["x"].to(F32) * c, 0.0)
        return {"y": (y if s["res"] is None else y + s["res"].to(F32)).to(TYPES[case["y"]])}
    # verify, in 64 bits: tests and samples lie next to borders
    n, k, V = case["n"], case["k"], case["V"]
    at = torch.arange(n, device="cuda")

    def log_softmax(z):
        z = z.to(F64) / case["temperature"]
        z = z - z.amax(1, keepdim=True)
        return z - torch.exp(z).sum(1, keepdim=True).log()

    lp = log_softmax(s["z"]).view(n, k + 1, V)
    ids, place = s["drafts"].long(), torch.arange(k, device="cuda")
    lens = torch.full((n,), k, device="cuda") if s["lens"] is None else s["lens"].long()
    p_draft = lp[:, :k].gather(2, ids[:, :, None])[:, :, 0].exp()
    lq = None if s["zd"] is None else log_softmax(s["zd"]).view(n, k, V)
    q_draft = torch.ones_like(p_draft) if lq is None else lq.gather(2, ids[:, :, None])[:, :, 0].exp()
    good = (s["u"][:, :k].to(F64) * q_draft < p_draft) & (place < lens[:, None])
    a = good.to(I64).cumprod(1).sum(1) if k else torch.zeros_like(lens)
    p = lp[at, a].exp()
    if k:
        b = a.clamp(max=k - 1)
        if lq is None:
            q = torch.zeros_like(p).scatter_(1, ids[at, b][:, None], 1.0)
        else:
            q = lq[at, b].exp()
        left = (p - torch.where((a < lens)[:, None], q, 0.0)).clamp(min=0.0)
        p = torch.where(left.sum(1, keepdim=True) > 0, left, p)
    to = p.cumsum(1)
    chosen = (to <= s["u"][:, k:].to(F64) * to[:, -1:]).sum(1).clamp(max=V - 1)
    place = torch.arange(k + 1, device="cuda")
    tokens = torch.where(place < a[:, None], torch.nn.functional.pad(ids, (0, 1)), -1)
    tokens[at, a] = chosen
    out = lp.gather(2, tokens.clamp(min=0)[:, :, None])[:, :, 0]
    return {"accepted": a.to(torch.int32), "tokens": tokens.to(torch.int32),
            "lp": torch.where(place <= a[:, None], out, 0.0).to(F32)}


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        M, K = case["M"], case["K"]
        copies = 2 if case["transposed"] else 1
        return {"bytes": M * K * (BYTES[case["x"]] + copies) + copies * _up(M, case["block_rows"]) * _up(K, BLOCK),
                "flops": 2 * M * K}
    if kind == "linear":
        M, N, K, r = case["M"], case["N"], case["K"], case["r"] if case["on"] else 0
        return {"bytes": 2 * M * K + N * K + _up(N, BLOCK) * _up(K, BLOCK) + 2 * r * (N + K)
                + M * N * BYTES[case["y"]] * (case["off"] + case["on"]), "flops": 2 * M * (N * K + r * (N + K))}
    if kind == "backward":
        M, N, K, r = case["M"], case["N"], case["K"], case["r"]
        return {"bytes": 2 * M * (K + N) + N * K + _up(N, BLOCK) * _up(K, BLOCK) + 6 * r * (N + K)
                + M * K * BYTES[case["dx"]], "flops": 2 * M * (N * K + 3 * r * (N + K) - r * N)}
    if kind == "dropout":
        res = 0 if case["res"] == "none" else BYTES[case["res"]]
        return {"bytes": case["M"] * case["K"] * (BYTES[case["x"]] + res + BYTES[case["y"]]),
                "flops": 2 * case["M"] * case["K"]}
    n, k, V = case["n"], case["k"], case["V"]
    zd = 0 if case["zd"] == "none" else BYTES[case["zd"]]
    return {"bytes": n * V * ((k + 1) * BYTES[case["z"]] + k * zd) + 4 * n * (4 * k + 4), "flops": 6 * n * V * (2 * k + 1)}


def _exact_quantize(x, rows):
    """The nearest of the type's values, found among all of them, in 64 bits: (values in the scale's units, whole e)."""
    x = x.to(F64)
    M, K = x.shape
    x = torch.where(torch.isfinite(x), x, math.nan)
    a = _blocks(torch.nan_to_num(x, nan=0.0).abs(), rows).amax((1, 3))
    e = torch.ceil(torch.log2(a.clamp(min=2.0 ** -300) / 448))
    e = torch.where(a > 448 * torch.exp2(e), e + 1, torch.where(a <= 224 * torch.exp2(e), e - 1, e)).clamp(min=-127)
    code = torch.arange(127, device="cuda", dtype=F64)
    fraction, power = code % 8, torch.floor(code / 8)
    every = torch.where(power > 0, (1 + fraction / 8) * torch.exp2(power - 7), fraction * 2.0 ** -9)
    middle = (every[1:] + every[:-1]) / 2
    v = x * torch.exp2(-_spread(e, rows, M, K))
    i = torch.bucketize(v.abs().nan_to_num(nan=0.0), middle)
    tie = v.abs() == middle[i.clamp(max=125)]
    i = torch.where(tie & (i % 2 == 1), i + 1, i)
    return torch.where(torch.isnan(v), v, torch.copysign(every[i], v)), e


def _exact_values(x):
    q, e = _exact_quantize(x, 1)
    return q * torch.exp2(_spread(e, 1, *q.shape))


def _exact_weight(i):
    e = torch.exp2(i["ws"].to(F64) - 127)
    N, K = i["wq"].shape
    return i["wq"].to(F64) * e.repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)[:, :K]


def _exact_words(seed, offset, groups):
    """Philox4x32-10 over counters 0 .. groups - 1, in numpy's unsigned numbers: [groups, 8] of 16 bits."""
    import numpy as np
    u = np.uint64
    mask = u(0xFFFFFFFF)
    g = np.arange(groups, dtype=u)
    c = [g & mask, g >> u(32), np.full_like(g, offset & 0xFFFFFFFF), np.full_like(g, (offset >> 32) & 0xFFFFFFFF)]
    key = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        first, second = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(second >> u(32)) ^ c[1] ^ u(key[0]), second & mask, (first >> u(32)) ^ c[3] ^ u(key[1]), first & mask]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    return np.stack(c, 1).astype(np.uint32).view(np.uint16).reshape(groups, 8)


def _exact_factor(rng, p, M, K):
    """What each element is multiplied by."""
    seed, offset = (int(v) % (1 << 64) for v in rng.tolist())
    bits = _exact_words(seed, offset, _up(M * K, 8)).reshape(-1)[:M * K].reshape(M, K)
    dropped = round(p * 65536)
    keep = torch.from_numpy(bits >= dropped).cuda()
    return keep.to(F64) * (1.0 / (1.0 - dropped / 65536) if dropped < 65536 else 0.0)


def exact(case, seed):
    i, kind = _inputs(case, seed), case["kind"]
    if kind == "quantize":
        q, e = _exact_quantize(i["x"], case["block_rows"])
        t = case["transposed"]
        return {"q": q, "scale": None, "qt": q.t().contiguous() if t else None, "scale_t": None}
    if kind == "linear":
        y = torch.matmul(_exact_values(i["x"]), _exact_weight(i).t())
        x, A, B = (i[n].to(F64) for n in ("x", "A", "B"))
        return {"y_off": y if case["off"] else None,
                "y_on": torch.addmm(y, x @ A.t() * i["s"], B.t()) if case["on"] else None}
    if kind == "backward":
        x, dy, A, B = (i[n].to(F64) for n in ("x", "dy", "A", "B"))
        through = i["s"] * (dy @ (B @ A))
        if case["p"] > 0:
            through = through * _exact_factor(i["rng"], case["p"], case["M"], case["K"])
        return {"dx": _exact_values(i["dy"]) @ _exact_weight(i).t() + through, "dA": i["s"] * (B.t() @ (dy.t() @ x)),
                "dB": i["s"] * ((dy.t() @ x) @ A.t())}
    if kind == "dropout":
        y = i["x"].to(F64) * _exact_factor(i["rng"], case["p"], case["M"], case["K"])
        return {"y": y if i["res"] is None else y + i["res"].to(F64)}
    # one sequence at a time, in the order in which a program without drafts would go
    n, k, T = case["n"], case["k"], case["temperature"]
    u = i["u"].to(F64).tolist()
    drafts, lens = i["drafts"].tolist(), [k] * n if i["lens"] is None else i["lens"].tolist()
    lp = torch.zeros(n, k + 1, dtype=F64, device="cuda")
    for b in range(n):
        for j in range(lens[b] + 1):
            row = torch.log_softmax(i["z"][b * (k + 1) + j].to(F64) / T, 0)
            if j < lens[b]:
                t = drafts[b][j]
                if i["zd"] is None:
                    q = torch.nn.functional.one_hot(torch.tensor(t, device="cuda"), case["V"]).to(F64)
                else:
                    q = torch.softmax(i["zd"][b * k + j].to(F64) / T, 0)
                if u[b][j] * float(q[t]) < math.exp(float(row[t])):
                    lp[b, j] = row[t]
                    continue
                left = torch.relu(row.exp() - q)
            else:
                left = row.exp()
            sums = torch.cumsum(left, 0)
            lp[b, j] = row[int(torch.searchsorted(sums, u[b][k] * float(sums[-1]), right=True))]
            break
    return {"accepted": None, "tokens": None, "lp": lp}
