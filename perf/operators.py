"""The operators around the PPO losses and the linear's backward in an update step, as cases to time.

A case is a dict of plain values; "kind" names the entry point it goes through:

* norm       layer norm of a block of rows (hydra_layer_norm)
* norm_back  its gradients: rows, weight and bias (hydra_layer_norm_backward)
* logp       log-probabilities of given tokens with entropy and top alternatives (hydra_token_logprobs)
* logp_back  their gradient with respect to the logits (hydra_token_logprobs_backward)
* clip       the norm over many gradient tensors and the clipped gradients (hydra_grad_clip)

Sizes are those of the repository's Llama-7B and OPT-1.3b configurations (hidden 4096 and 2048, vocabulary 32000 and
50272, ranks 16 and 128, batches of 4 and 8 sequences of 512 tokens) and ragged ones between them.
"""
import math

import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
TYPES = {"bf16": BF16, "f32": F32}
BYTES = {"bf16": 2, "f32": 4}
EPS = 1e-5
WORKSPACE = 32 << 20  # bytes of scratch memory that a program keeps for whichever call comes

# (K, N) of the linears of one layer: q, k, v, o, then the MLP
LLAMA = [(4096, 4096)] * 4 + [(4096, 11008)] * 2 + [(11008, 4096)]
OPT = [(2048, 2048)] * 4 + [(2048, 8192), (8192, 2048)]


def listed():
    return [
        # one token for each of 4 sequences in a generation step: latency alone
        dict(name="norm_token", kind="norm", M=4, K=2048, x="bf16", w="bf16", y="bf16"),
        # OPT-1.3b's mini-batch of 8 x 512 tokens, the fp32 residual stream into the bf16 rows that a linear reads
        dict(name="norm_batch", kind="norm", M=4096, K=2048, x="f32", w="bf16", y="bf16"),
        # the same mini-batch's backward: the linear's fp32 dx comes in
        dict(name="norm_back_batch", kind="norm_back", M=4096, K=2048, dy="f32", x="f32", w="bf16", dx="f32"),
        # one ragged sequence, everything in bf16
        dict(name="norm_back_sequence", kind="norm_back", M=333, K=4096, dy="bf16", x="bf16", w="bf16", dx="bf16"),
        # a generation step of 6 sequences over OPT-1.3b's vocabulary, eight alternatives with each token
        dict(name="logp_token", kind="logp", M=6, V=50272, z="f32", top=8, masked=0.0),
        # actor log-probabilities and entropy of a batch of 4 x 512 tokens, Llama-7B vocabulary
        dict(name="logp_batch", kind="logp", M=2048, V=32000, z="f32", top=0, masked=0.0),
        # an evaluation over a program's own bf16 logits, the twenty best of each, a tenth of the vocabulary masked out
        dict(name="logp_top", kind="logp", M=1000, V=32000, z="bf16", top=20, masked=0.1),
        # the update stage: 4 x 512 tokens, half of them prompt, into the bf16 dy of the head's backward
        dict(name="logp_back_batch", kind="logp_back", n_seq=4, seq_len=512, start=256, V=32000, z="f32", dz="bf16",
             entropy=False),
        # one sequence with an entropy bonus over OPT-1.3b's vocabulary
        dict(name="logp_back_sequence", kind="logp_back", n_seq=1, seq_len=250, start=37, V=50272, z="bf16", dz="bf16",
             entropy=True),
        # the adapters of one attention block at rank 16: eight small tensors
        dict(name="clip_block", kind="clip", model="opt", layers=1, linears=4, r=16, g="f32", out="f32", max_norm=1.0),
        # every adapter of Llama-7B at rank 16, 448 tensors, into the bf16 bucket of a collective
        dict(name="clip_llama", kind="clip", model="llama", layers=32, linears=7, r=16, g="f32", out="bf16", max_norm=1.0),
        # every adapter of OPT-1.3b at the paper's rank 128, 288 tensors
        dict(name="clip_opt_r128", kind="clip", model="opt", layers=24, linears=6, r=128, g="f32", out="f32", max_norm=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_back", "logp", "logp", "logp_back", "clip"])

    def t():
        return rng.choice(["bf16", "f32"])

    if kind in ("norm", "norm_back"):
        K = rng.choice([2048, 4096, 8 * _log(rng, 16, 1376), _log(rng, 65, 11008)])
        M = min(_log(rng, 1, 16384), (1 << 25) // K)
        if kind == "norm":
            return dict(kind=kind, M=M, K=K, x=t(), w=t(), y=t())
        return dict(kind=kind, M=M, K=K, dy=t(), x=t(), w=t(), dx=t())
    V = rng.choice([32000, 50272, _log(rng, 1000, 60000), 2 * _log(rng, 500, 30000)])
    top = 2048 * 32000 // V
    if kind == "logp":
        return dict(kind=kind, M=min(_log(rng, 1, 4096), top), V=V, z=t(), top=rng.choice([0, 1, 5, 8, 20, 32]),
                    masked=rng.choice([0.0, 0.0, 0.1, 0.9]))
    if kind == "logp_back":
        seq_len = _log(rng, 1, 1024)
        return dict(kind=kind, n_seq=max(1, min(_log(rng, 1, 8), top // seq_len)), seq_len=seq_len,
                    start=rng.randrange(seq_len), V=V, z=t(), dz=t(), entropy=rng.random() < 0.5)
    model = rng.choice(["llama", "opt"])
    r = rng.choice([8, 16, 64, 128, rng.randrange(1, 129)])
    most = 32 if model == "llama" else 24
    per_layer = r * sum(K + N for K, N in (LLAMA if model == "llama" else OPT))
    return dict(kind=kind, model=model, layers=min(_log(rng, 1, most), max(1, 100_000_000 // per_layer)),
                linears=rng.choice([2, 4, 6]), r=r, g=t(), out=t(), max_norm=rng.choice([0.5, 1.0, 1e6]))


def _sizes(case):
    """The adapters' gradient tensors: A [r x K] and B [N x r] of each linear."""
    r, sizes = case["r"], []
    for K, N in (LLAMA if case["model"] == "llama" else OPT)[:case["linears"]] * case["layers"]:
        sizes += [(r, K), (N, r)]
    return sizes


class _Draw:
    """Seeded tensors on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, *shape, std=1.0, mean=0.0, dtype=F32):
        return torch.randn(*shape, generator=self.g, device="cuda", dtype=F32).mul_(std).add_(mean).to(dtype)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda", dtype=F32)


def _inputs(case, seed):
    d, kind, i = _Draw(seed), case["kind"], {}
    if kind in ("norm", "norm_back"):
        M, K = case["M"], case["K"]
        # hidden states with channels of their own mean and width
        i["x"] = (d.normal(M, K) * (0.5 + 2 * d.uniform(K)) + d.normal(K, std=0.3)).to(TYPES[case["x"]])
        i["w"] = d.normal(K, std=0.2, mean=1.0, dtype=TYPES[case["w"]])
        i["b"] = d.normal(K, std=0.1, dtype=TYPES[case["w"]])
        if kind == "norm_back":
            x = i["x"].to(F64)
            i["mean"] = x.mean(1).to(F32)
            i["rstd"] = (x.var(1, unbiased=False) + EPS).rsqrt().to(F32)
            i["dy"] = d.normal(M, K, std=1e-2, dtype=TYPES[case["dy"]])
        return i
    if kind in ("logp", "logp_back"):
        V = case["V"]
        M = case["M"] if kind == "logp" else case["n_seq"] * case["seq_len"]
        z = d.normal(M, V, std=2.0)
        if case.get("masked"):
            z.masked_fill_(d.uniform(M, V) < case["masked"], -math.inf)
        i["z"] = z.to(TYPES[case["z"]])
        # tokens sampled from the distribution itself: the largest of z plus Gumbel noise
        noise = d.uniform(M, V).clamp_(1e-9, 1 - 1e-7).log_().neg_().log_().neg_()
        i["tokens"] = noise.add_(z).argmax(1).to(torch.int32)
        if kind == "logp_back":
            zz = i["z"].to(F64) if M * V <= 1 << 25 else i["z"].to(F32)
            lse = torch.logsumexp(zz, 1)
            i["lse"] = lse.to(F32)
            i["entropy"] = (lse - (torch.exp(zz - lse[:, None]) * zz).sum(1)).to(F32)
            response = (torch.arange(case["seq_len"], device="cuda") >= case["start"]).repeat(case["n_seq"])
            n = case["n_seq"] * (case["seq_len"] - case["start"])
            i["d_lp"] = d.normal(M, std=1.0 / n) * response
            i["d_entropy"] = response * (-0.01 / n) if case["entropy"] else None
        return i
    # gradients of different sizes from layer to layer
    i["g"] = [d.normal(*s, std=1e-3 * (1 + k % 5), dtype=TYPES[case["g"]]) for k, s in enumerate(_sizes(case))]
    return i


def prepare(case, seed):
    """The inputs, and the output buffers and workspace that a program allocates once."""
    s = _inputs(case, seed)
    s["case"], kind = case, case["kind"]

    def out(*shape, dtype=F32):
        return torch.empty(shape, device="cuda", dtype=dtype)

    if kind == "norm":
        M, K = case["M"], case["K"]
        s["y"], s["mean"], s["rstd"] = out(M, K, dtype=TYPES[case["y"]]), out(M), out(M)
    elif kind == "norm_back":
        M, K = case["M"], case["K"]
        s["dx"], s["dw"], s["db"] = out(M, K, dtype=TYPES[case["dx"]]), out(K), out(K)
    elif kind == "logp":
        M, top = case["M"], case["top"]
        s["lp"], s["lse"], s["entropy"] = out(M), out(M), out(M)
        s["ids"] = out(M, top, dtype=torch.int32) if top else None
        s["top_lp"] = out(M, top) if top else None
    elif kind == "logp_back":
        s["dz"] = out(case["n_seq"] * case["seq_len"], case["V"], dtype=TYPES[case["dz"]])
    else:
        # the clipped gradients go into one flat bucket
        n = [g.numel() for g in s["g"]]
        s["flat"] = out(sum(n), dtype=TYPES[case["out"]])
        s["out"] = [f.view(g.shape) for f, g in zip(s["flat"].split(n), s["g"])]
        s["norm"] = out(1)
    s["ws"] = out(WORKSPACE, dtype=torch.uint8)
    return s


def _outputs(s):
    names = {"norm": ("y", "mean", "rstd"), "norm_back": ("dx", "dw", "db"),
             "logp": ("lp", "lse", "entropy", "ids", "top_lp"), "logp_back": ("dz",), "clip": ("norm", "flat")}
    return {k: s[k] for k in names[s["case"]["kind"]]}


def _run_own(s):
    import paper_2309_00754_amd as H
    kind = s["case"]["kind"]
    if kind == "norm":
        H.hydra_layer_norm(s["x"], s["w"], s["b"], s["y"], s["mean"], s["rstd"], eps=EPS)
    elif kind == "norm_back":
        H.hydra_layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"], s["ws"])
    elif kind == "logp":
        H.hydra_token_logprobs(s["z"], s["tokens"], s["lp"], s["lse"], s["entropy"], s["ids"], s["top_lp"], s["ws"])
    elif kind == "logp_back":
        H.hydra_token_logprobs_backward(s["z"], s["tokens"], s["lse"], s["dz"], s["d_lp"], s["entropy"], s["d_entropy"])
    else:
        H.hydra_grad_clip(s["g"], s["case"]["max_norm"], s["norm"], s["out"], s["ws"])
    return _outputs(s)


def _best(z, k):
    """Indices of the k largest of each row, the lowest first among equals: one whole number per logit that orders by value,
    then by index."""
    V = z.shape[1]
    bits = (z + 0.0).view(torch.int32)
    bits = bits ^ ((bits >> 31) & 0x7FFFFFFF)
    key = bits.to(torch.int64) * (1 << 32) + (V - 1 - torch.arange(V, device=z.device))
    return V - 1 - (torch.topk(key, k, dim=1).values & 0xFFFFFFFF)


def run(s):
    if own:
        return _run_own(s)
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        x = s["x"].to(F32)
        mean = x.sum(1, keepdim=True) / case["K"]
        c = x - mean
        rstd = ((c * c).sum(1, keepdim=True) / case["K"] + EPS).rsqrt()
        return {"y": (c * rstd * s["w"].to(F32) + s["b"].to(F32)).to(TYPES[case["y"]]), "mean": mean[:, 0],
                "rstd": rstd[:, 0]}
    if kind == "norm_back":
        K, dy, rstd = case["K"], s["dy"].to(F32), s["rstd"][:, None]
        xh = (s["x"].to(F32) - s["mean"][:, None]) * rstd
        g = dy * s["w"].to(F32)
        dx = rstd * (g - g.sum(1, keepdim=True) / K - xh * ((g * xh).sum(1, keepdim=True) / K))
        return {"dx": dx.to(TYPES[case["dx"]]), "dw": (dy * xh).sum(0), "db": dy.sum(0)}
    if kind == "logp":
        z = s["z"].to(F32)
        most = z.amax(1, keepdim=True)
        c = z - most
        e = torch.exp(c)
        total = e.sum(1, keepdim=True)
        lse = total.log() + most
        mean_c = torch.where(e > 0, e * c, 0.0).sum(1, keepdim=True) / total
        ids = _best(z, case["top"]) if case["top"] else None
        return {"lp": (z.gather(1, s["tokens"].long()[:, None]) - lse)[:, 0], "lse": lse[:, 0],
                "entropy": (total.log() - mean_c)[:, 0], "ids": None if ids is None else ids.to(torch.int32),
                "top_lp": None if ids is None else z.gather(1, ids) - lse}
    if kind == "logp_back":
        lp = s["z"].to(F32) - s["lse"][:, None]
        p = torch.exp(lp)
        f = -s["d_lp"][:, None]
        if s["d_entropy"] is not None:
            f = f - s["d_entropy"][:, None] * (lp + s["entropy"][:, None])
        dz = p * f
        dz.scatter_add_(1, s["tokens"].long()[:, None], s["d_lp"][:, None])
        return {"dz": dz.to(TYPES[case["dz"]])}
    flat = torch.cat([g.reshape(-1) for g in s["g"]])
    norm = flat.to(F64).square().sum().sqrt()  # in 64 bits: a hundred million terms
    coef = torch.where(norm > case["max_norm"], case["max_norm"] / norm, 1.0).to(F32)
    return {"norm": norm.to(F32).reshape(1), "flat": (flat.to(F32) * coef).to(TYPES[case["out"]])}


def work(case):
    kind = case["kind"]
    if kind == "norm":
        M, K = case["M"], case["K"]
        return {"bytes": M * K * (BYTES[case["x"]] + BYTES[case["y"]]) + 2 * K * BYTES[case["w"]] + 8 * M,
                "flops": 8 * M * K}
    if kind == "norm_back":
        M, K = case["M"], case["K"]
        return {"bytes": M * K * (BYTES[case["dy"]] + BYTES[case["x"]] + BYTES[case["dx"]]) + K * BYTES[case["w"]] + 8 * K
                + 8 * M, "flops": 16 * M * K}
    if kind == "logp":
        M, V = case["M"], case["V"]
        return {"bytes": M * V * BYTES[case["z"]] + M * (16 + 8 * case["top"]), "flops": 6 * M * V}
    if kind == "logp_back":
        M, n = case["n_seq"] * case["seq_len"], case["n_seq"] * (case["seq_len"] - case["start"])
        # a prompt token's gradient is zero: its logits need not be read
        return {"bytes": n * case["V"] * BYTES[case["z"]] + M * case["V"] * BYTES[case["dz"]] + 16 * M,
                "flops": 6 * n * case["V"]}
    n = sum(a * b for a, b in _sizes(case))
    return {"bytes": n * (BYTES[case["g"]] + BYTES[case["out"]]) + 4, "flops": 3 * n}


def _exact_logp(z, tokens, top):
    """One block of rows in 64 bits."""
    z = z.to(F64) + 0.0
    lse = torch.logsumexp(z, 1)
    lp = z - lse[:, None]
    p = lp.exp()
    o = {"lp": lp.gather(1, tokens.long()[:, None])[:, 0], "lse": lse,
         "entropy": -(p * lp).masked_fill(p == 0, 0.0).sum(1), "ids": None, "top_lp": None}
    if top:
        v, at = torch.sort(lp, dim=1, descending=True, stable=True)
        o["ids"], o["top_lp"] = at[:, :top].to(torch.int32), v[:, :top]
    return o


def exact(case, seed):
    i, kind = _inputs(case, seed), case["kind"]
    if kind == "norm":
        x = i["x"].to(F64)
        var, mean = torch.var_mean(x, 1, unbiased=False)
        rstd = 1.0 / torch.sqrt(var + EPS)
        return {"y": (x - mean[:, None]) / torch.sqrt(var + EPS)[:, None] * i["w"].to(F64) + i["b"].to(F64), "mean": mean,
                "rstd": rstd}
    if kind == "norm_back":
        dy, x, w, mean, rstd = (i[k].to(F64) for k in ("dy", "x", "w", "mean", "rstd"))
        xh = (x - mean[:, None]) * rstd[:, None]
        g = dy * w
        dx = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * rstd[:, None]
        return {"dx": dx, "dw": torch.einsum("mk,mk->k", dy, xh), "db": dy.mean(0) * case["M"]}
    if kind == "logp":
        blocks = [_exact_logp(i["z"][m:m + 128], i["tokens"][m:m + 128], case["top"]) for m in range(0, case["M"], 128)]
        return {k: None if blocks[0][k] is None else torch.cat([b[k] for b in blocks]) for k in blocks[0]}
    if kind == "logp_back":
        dz = []
        for m in range(0, len(i["tokens"]), 128):
            rows = slice(m, m + 128)
            lp = i["z"][rows].to(F64) - i["lse"][rows].to(F64)[:, None]
            chosen = torch.nn.functional.one_hot(i["tokens"][rows].long(), case["V"])
            d = i["d_lp"][rows].to(F64)[:, None] * (chosen - lp.exp())
            if i["d_entropy"] is not None:
                h = i["entropy"][rows].to(F64)[:, None]
                d -= i["d_entropy"][rows].to(F64)[:, None] * lp.exp() * (lp + h)
            dz.append(d)
        return {"dz": torch.cat(dz)}
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(g.to(F64))) ** 2 for g in i["g"]))
    scale = min(1.0, case["max_norm"] / norm)
    return {"norm": torch.tensor([norm], dtype=F64), "flat": torch.cat([g.reshape(-1).to(F64) * scale for g in i["g"]])}
