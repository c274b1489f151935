"""Workloads of the 8-bit language-model operators: the norm and the gate that quantise, the scaled product, token scores.

Each case is one call as a program makes it.  With ``own`` false the operators are computed by elementary torch
operations in fp32, rounded once at the end; with ``own`` true by the library.  Codes held in 8 bits are returned as the
values they stand for (code times scale), which the quantising calls can write next to the codes.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def listed():
    return [
        # the norm before a block's products, one token being generated: latency is all
        {"name": "norm_one_token", "op": "norm", "rows": 1, "K": 4096, "type": "bf16", "residual": True},
        # the same over a long prompt
        {"name": "norm_prompt", "op": "norm", "rows": 8192, "K": 4096, "type": "bf16", "residual": True},
        # the gated activation between a block's two products: a small batch of single tokens
        {"name": "gate_tokens", "op": "gate", "rows": 8, "K": 11000, "type": "bf16"},
        # over a prompt, in half precision
        {"name": "gate_prompt", "op": "gate", "rows": 4096, "K": 12288, "type": "f16"},
        # one token through a square layer: the weights' bytes are the cost
        {"name": "product_one_token", "op": "product", "M": 1, "N": 4096, "K": 4096, "type": "bf16", "bias": False},
        # a batch of 100 through the 4096-unit layer
        {"name": "product_batch", "op": "product", "M": 100, "N": 4096, "K": 4096, "type": "f16", "bias": False},
        # odd sizes, a bias, fp32 results
        {"name": "product_odd", "op": "product", "M": 701, "N": 2047, "K": 1111, "type": "f32", "bias": True},
        # a prompt of 10000 tokens through the 4096-unit layer
        {"name": "product_prompt", "op": "product", "M": 10000, "N": 4096, "K": 4096, "type": "bf16", "bias": False},
        # scores of four tokens being generated, with the five best alternatives
        {"name": "scores_tokens", "op": "scores", "T": 4, "V": 128000, "type": "bf16", "top": 5, "masked": 0},
        # scores of a training batch over a large vocabulary whose padding is masked
        {"name": "scores_batch", "op": "scores", "T": 2048, "V": 131072, "type": "bf16", "top": 8, "masked": 1072},
        # gradient of log probability and entropy: a short sequence in fp32, an odd vocabulary
        {"name": "scores_grad_short", "op": "scores_grad", "T": 33, "V": 50021, "type": "f32", "masked": 0},
        # and a training batch
        {"name": "scores_grad_batch", "op": "scores_grad", "T": 2048, "V": 131072, "type": "bf16", "masked": 1072},
    ]


def _log_size(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, max(lo, n))


def _width(rng, lo, hi):
    # widths are mostly whole vectors, as in real models; one in four is whatever comes
    n = _log_size(rng, lo, hi)
    return n if rng.random() < 0.25 else max(lo, n // 64 * 64)


def draw(rng):
    op = rng.choice(["norm", "gate", "product", "product", "scores", "scores_grad"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "norm":
        K = _width(rng, 256, 16384)
        rows = _log_size(rng, 1, max(1, min(16384, 8192 * 4096 // K)))
        return {"op": op, "rows": rows, "K": K, "type": kind, "residual": rng.random() < 0.75}
    if op == "gate":
        K = _width(rng, 512, 28672)
        rows = _log_size(rng, 1, max(1, min(16384, 4096 * 12288 // K)))
        return {"op": op, "rows": rows, "K": K, "type": kind}
    if op == "product":
        N, K = _width(rng, 128, 16384), _width(rng, 128, 16384)
        most = 10000 * 4096 * 4096 // (N * K)
        return {"op": op, "M": _log_size(rng, 1, max(1, min(10000, most))), "N": N, "K": K, "type": kind,
                "bias": rng.random() < 0.5}
    V = _width(rng, 1000, 131072)
    T = _log_size(rng, 1, max(1, min(8192, 2048 * 131072 // (V * (2 if kind == "f32" else 1)))))
    case = {"op": op, "T": T, "V": V, "type": kind, "masked": rng.choice([0, 0, V // 100])}
    if op == "scores":
        case["top"] = rng.choice([0, 1, 5, 8, 20])
    return case


def _pitch(K):
    return (K + 127) // 128 * 128        # rows of 8-bit operands start on whole 128-byte lines


def _codes(x):
    """Rows of fp32 -> int8 codes (rows a whole number of lines apart, pads zero) and scales."""
    rows, K = x.shape
    top = x.abs().amax(1)
    q = torch.zeros(rows, _pitch(K), dtype=torch.int8, device=x.device)
    q[:, :K] = torch.round(x * (127.0 / top)[:, None]).to(torch.int8)
    return q, top / 127.0


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    s = dict(case)
    dt = TYPES[case["type"]]
    s["dt"] = dt
    if case["op"] == "norm":
        rows, K = case["rows"], case["K"]
        # activations with a few strong channels, as residual streams have them
        strength = torch.exp(0.8 * normal(K))
        s["x"] = (normal(rows, K) * 0.5).to(dt)
        s["residual"] = (normal(rows, K) * strength).to(dt) if case["residual"] else None
        s["gamma"] = (1.0 + 0.2 * normal(K)).to(dt)
        s["sum"] = torch.empty(rows, K, dtype=dt, device=dev) if case["residual"] else None
    elif case["op"] == "gate":
        rows, K = case["rows"], case["K"]
        both = (normal(rows, 2 * K) * 1.5).to(dt)        # one product gives gate and up side by side
        s["gate"], s["up"] = both[:, :K], both[:, K:]
    if case["op"] in ("norm", "gate"):
        s["codes"] = torch.empty(rows, _pitch(K), dtype=torch.int8, device=dev)
        s["scale"] = torch.empty(rows, dtype=torch.float32, device=dev)
        # a code is one of 255 values: 16 bits hold what it stands for, whatever the input's type
        s["values"] = torch.empty(rows, K, dtype=torch.bfloat16 if dt == torch.float32 else dt, device=dev)
    elif case["op"] == "product":
        M, N, K = case["M"], case["N"], case["K"]
        s["a"], s["a_scale"] = _codes(normal(M, K))
        s["b"], s["b_scale"] = _codes(normal(N, K) / math.sqrt(K))
        s["bias_v"] = normal(N) * 0.1 if case["bias"] else None
        s["out"] = torch.empty(M, N, dtype=dt, device=dev)
    elif case["op"] in ("scores", "scores_grad"):
        T, V = case["T"], case["V"]
        z = (normal(T, V) * 2.5).to(dt)
        if case["masked"]:
            z[:, V - case["masked"]:] = float("-inf")
        s["logits"] = z
        s["ids"] = torch.randint(0, V - case["masked"], (T,), generator=g, device=dev)
        if case["op"] == "scores":
            k = case["top"]
            s["logprob"], s["entropy"], s["lse"] = (torch.empty(T, device=dev) for _ in range(3))
            s["top_logprob"] = torch.empty(T, k, device=dev) if k else None
            s["top_ids"] = torch.empty(T, k, dtype=torch.int64, device=dev) if k else None
        else:
            # what the forward pass left, and the gradients that come back
            zf = z.float()
            s["lse"] = torch.logsumexp(zf, 1)
            p = torch.exp(zf - s["lse"][:, None])
            s["entropy"] = s["lse"] - torch.where(p > 0, p * zf, torch.zeros_like(p)).sum(1)
            s["g_logprob"], s["g_entropy"] = normal(T), normal(T) * 0.1
            s["grad"] = torch.empty(T, V, dtype=dt, device=dev)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------

def _plain_quantised(t, norm, dt):
    top = t.abs().amax(1)
    scale = top * norm / 127.0
    code = torch.round(t * (127.0 / top)[:, None])
    return scale, (code * scale[:, None]).to(dt)


def _plain(s):
    op, dt = s["op"], s["dt"]
    if op == "norm":
        h = s["x"].float()
        if s["residual"] is not None:
            h = h + s["residual"].float()
        norm = 1.0 / torch.sqrt((h * h).mean(1) + EPS)
        scale, values = _plain_quantised(h * s["gamma"].float(), norm, s["values"].dtype)
        out = {"scale": scale, "values": values}
        if s["residual"] is not None:
            out["sum"] = h.to(dt)
        return out
    if op == "gate":
        a = s["gate"].float()
        y = a / (1.0 + torch.exp(-a)) * s["up"].float()
        scale, values = _plain_quantised(y, 1.0, s["values"].dtype)
        return {"scale": scale, "values": values}
    if op == "product":
        K = s["K"]
        y = torch.matmul(s["a"][:, :K].float(), s["b"][:, :K].float().t())
        y = y * s["a_scale"][:, None] * s["b_scale"][None, :]
        if s["bias_v"] is not None:
            y = y + s["bias_v"]
        return {"out": y.to(dt)}
    z = s["logits"].float()
    if op == "scores":
        m = z.amax(1, keepdim=True)
        e = torch.exp(z - m)
        total = e.sum(1)
        lse = m[:, 0] + torch.log(total)
        away = torch.where(e > 0, z - m, torch.zeros_like(z))
        out = {"logprob": z.gather(1, s["ids"][:, None])[:, 0] - lse, "lse": lse,
               "entropy": torch.log(total) - (e * away).sum(1) / total}
        if s["top"]:
            # one whole number an element that orders by value first and by the lower index next
            b = z.view(torch.int32)
            order = torch.where(b < 0, b ^ 0x7FFFFFFF, b).to(torch.int64)
            order = order * (1 << 32) + (s["V"] - torch.arange(s["V"], device=z.device))
            top_ids = torch.topk(order, s["top"], dim=1).indices
            out["top_ids"] = top_ids
            out["top_logprob"] = z.gather(1, top_ids) - lse[:, None]
        return out
    logp = z - s["lse"][:, None]
    p = torch.exp(logp)
    away = torch.where(p > 0, logp, torch.zeros_like(logp)) + s["entropy"][:, None]
    d = -p * (s["g_logprob"][:, None] + s["g_entropy"][:, None] * away)
    d.scatter_add_(1, s["ids"][:, None], s["g_logprob"][:, None])
    return {"grad": d.to(dt)}


# ---- the library -------------------------------------------------------------------------------------------------

def _own(s):
    from paper_1609_07061_b200 import binding as q
    op = s["op"]
    if op == "norm":
        K = s["K"]
        q.qnn_rmsnorm_quant_i8(s["x"], s["residual"], s["rows"], K, K, K, s["gamma"], EPS, s["codes"], s["codes"].shape[1],
                               s["scale"], sum_out=s["sum"], ld_sum=K, values=s["values"], ld_values=K)
        out = {"scale": s["scale"], "values": s["values"]}
        if s["residual"] is not None:
            out["sum"] = s["sum"]
        return out
    if op == "gate":
        K = s["K"]
        q.qnn_silu_mul_quant_i8(s["gate"], s["up"], s["rows"], K, 2 * K, 2 * K, s["codes"], s["codes"].shape[1], s["scale"],
                                values=s["values"], ld_values=K)
        return {"scale": s["scale"], "values": s["values"]}
    if op == "product":
        q.qnn_gemm_i8_scaled(s["a"], s["a"].shape[1], s["a_scale"], s["b"], s["b"].shape[1], s["b_scale"], s["M"], s["N"],
                             s["K"], s["out"], s["N"], bias=s["bias_v"])
        return {"out": s["out"]}
    T, V = s["T"], s["V"]
    if op == "scores":
        q.qnn_token_logprobs(s["logits"], T, V, V, s["ids"], s["logprob"], entropy=s["entropy"], lse=s["lse"],
                             topk=s["top"], top_logprob=s["top_logprob"], top_ids=s["top_ids"])
        out = {"logprob": s["logprob"], "lse": s["lse"], "entropy": s["entropy"]}
        if s["top"]:
            out["top_ids"], out["top_logprob"] = s["top_ids"], s["top_logprob"]
        return out
    q.qnn_token_logprobs_backward(s["logits"], T, V, V, s["ids"], s["lse"], s["entropy"], s["g_logprob"], s["g_entropy"],
                                  s["grad"], V)
    return {"grad": s["grad"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    es = 4 if case["type"] == "f32" else 2
    op = case["op"]
    if op == "norm":
        n = case["rows"] * case["K"]
        # x, the residual and its sum; codes and values; gamma, scales
        return {"bytes": n * (es * (3 if case["residual"] else 1) + 1 + 2) + case["K"] * es + case["rows"] * 4, "flops": 8.0 * n}
    if op == "gate":
        n = case["rows"] * case["K"]
        return {"bytes": n * (es * 2 + 1 + 2) + case["rows"] * 4, "flops": 8.0 * n}
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K + N * K + es * M * N + 4 * (M + N) + (4 * N if case["bias"] else 0), "flops": 2.0 * M * N * K}
    n = case["T"] * case["V"]
    if op == "scores":
        return {"bytes": n * es + case["T"] * (8 + 12 + 12 * case["top"]), "flops": 6.0 * n}
    return {"bytes": 2 * n * es + case["T"] * 24, "flops": 8.0 * n}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    f64 = torch.float64
    if op in ("norm", "gate"):
        if op == "norm":
            total = s["x"].to(f64) if s["residual"] is None else s["x"].to(f64).add_(s["residual"])
            y = total * s["gamma"].to(f64) / (total.square().mean(dim=1, keepdim=True) + EPS).sqrt()
        else:
            y = s["gate"].to(f64) * torch.sigmoid(s["gate"].to(f64)) * s["up"].to(f64)
        step = y.abs().max(dim=1, keepdim=True).values / 127
        out = {"scale": step[:, 0], "values": (y / step).round() * step}
        if op == "norm" and s["residual"] is not None:
            out["sum"] = total
        return out
    if op == "product":
        K = case["K"]
        # whole numbers below 2^53: exact in doubles
        y = s["a"][:, :K].to(f64) @ s["b"][:, :K].to(f64).T
        y *= s["a_scale"].to(f64).unsqueeze(1)
        y *= s["b_scale"].to(f64)
        if s["bias_v"] is not None:
            y += s["bias_v"].to(f64)
        return {"out": y}
    z = s["logits"].to(f64)
    rows = torch.arange(case["T"], device=z.device)
    logp = torch.log_softmax(z, dim=1)
    if op == "scores":
        out = {"logprob": logp[rows, s["ids"]], "lse": torch.logsumexp(z, dim=1), "entropy": torch.special.entr(logp.exp()).sum(1)}
        if case["top"]:
            out["top_ids"] = None
            out["top_logprob"] = torch.topk(logp, case["top"], dim=1).values
        return out
    # the derivative through a softmax: p * (c - <p, c>) for the cotangent c of log p, on the definition of the entropy
    p = logp.exp()
    c = torch.where(p > 0, -(logp + 1.0), torch.zeros_like(p)) * s["g_entropy"].to(f64)[:, None]
    grad = p * (c - (p * c).sum(1, keepdim=True))
    grad -= p * s["g_logprob"].to(f64)[:, None]
    grad[rows, s["ids"]] += s["g_logprob"].to(f64)
    return {"grad": grad}
