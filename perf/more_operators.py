"""Workloads of the operators on 8-bit floating point with a scale for each block of 128: the quantisers, the product and its
input gradient, the same grouped by expert, and the weight gradient.

A code (e4m3, for gradients also e5m2) stands for code * 2^(s - 127), s the byte of its block: 128 elements of a row of
activations, 128 x 128 of weights, 128 rows of a column for the operands of a weight gradient.  Each case is one call as a
program makes it.  With ``own`` false the operators are computed by elementary torch operations in fp32, rounded once at the
end; with ``own`` true by the library.  The quantisers' codes are returned as the values they stand for, which the calls can
write next to the codes, and the scales as their bytes.
"""
from __future__ import annotations

import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": (8, 448.0), "e5m2": (15, 57344.0)}         # exponent of the largest code, and its value
B = 128


def listed():
    return [
        # activations before a product, one token being generated: latency is all
        {"name": "rows_one_token", "op": "rows", "rows": 1, "K": 4096, "type": "bf16", "codes": "e4m3", "from": 0},
        # a prompt's tokens, each sent to four experts: rows quantised in the experts' order
        {"name": "rows_to_experts", "op": "rows", "rows": 16384, "K": 2048, "type": "bf16", "codes": "e4m3", "from": 4096},
        # weights of a layer, once each training step
        {"name": "tiles_weights", "op": "tiles", "rows": 11008, "K": 4096, "type": "f32", "codes": "e4m3"},
        # gradients of a training step, in blocks of tokens of one expert
        {"name": "columns_experts", "op": "columns", "rows": 16384, "K": 4096, "type": "bf16", "codes": "e5m2", "groups": 32, "skew": 1.0},
        # one token through a square layer: the weights' bytes are the cost
        {"name": "product_one_token", "op": "product", "M": 1, "N": 4096, "K": 4096, "type": "bf16", "codes": "e4m3", "back": False,
         "bias": False},
        # a batch whose sizes fit nothing, fp32 results, a bias
        {"name": "product_odd", "op": "product", "M": 701, "N": 2047, "K": 1111, "type": "f32", "codes": "e4m3", "back": False, "bias": True},
        # a prompt of 10000 tokens through the 4096-unit layer
        {"name": "product_prompt", "op": "product", "M": 10000, "N": 4096, "K": 4096, "type": "bf16", "codes": "e4m3", "back": False,
         "bias": False},
        # input gradient of a layer with a wide output, gradients in e5m2
        {"name": "product_input_gradient", "op": "product", "M": 4096, "N": 4096, "K": 11008, "type": "bf16", "codes": "e5m2", "back": True,
         "bias": False},
        # 16 tokens being generated, four experts of 64 each: most experts get one row or none
        {"name": "grouped_tokens", "op": "grouped", "M": 64, "N": 2816, "K": 2048, "type": "bf16", "codes": "e4m3", "back": False,
         "groups": 64, "skew": 0.5},
        # a prompt of 4096 tokens, four experts each of 32, some much sought
        {"name": "grouped_prompt", "op": "grouped", "M": 16384, "N": 4096, "K": 2048, "type": "f16", "codes": "e4m3", "back": False,
         "groups": 32, "skew": 1.0},
        # a small batch's weight gradient over odd sizes, in fp32
        {"name": "weight_gradient_odd", "op": "wgrad", "M": 1500, "N": 1000, "K": 2040, "type": "f32", "codes": "e4m3", "groups": 3, "skew": 1.0},
        # weight gradients of a training step's experts
        {"name": "weight_gradient_experts", "op": "wgrad", "M": 16384, "N": 4096, "K": 2048, "type": "bf16", "codes": "e5m2", "groups": 32,
         "skew": 1.0},
    ]


def _log_size(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return min(hi, max(lo, n))


def _width(rng, lo, hi):
    # widths are mostly whole vectors, as in real models; one in four is whatever comes
    n = _log_size(rng, lo, hi)
    return n if rng.random() < 0.25 else max(lo, n // 64 * 64)


def draw(rng):
    op = rng.choice(["rows", "tiles", "columns", "product", "product", "grouped", "grouped", "wgrad"])
    kind = rng.choice(["bf16", "bf16", "f16", "f32"])
    codes = rng.choice(["e4m3", "e4m3", "e5m2"])
    case = {"op": op, "type": kind, "codes": codes}
    if op in ("rows", "tiles", "columns"):
        K = _width(rng, 128, 16384)
        rows = _log_size(rng, 1, max(1, min(32768, 11008 * 4096 // K)))
        case.update(rows=rows, K=K)
        if op == "rows":
            case["from"] = 0 if rng.random() < 0.5 else max(1, rows // 4)
        elif op == "columns":
            case.update(groups=_log_size(rng, 1, 64), skew=rng.choice([0.0, 0.5, 1.0, 2.0]))
        return case
    N, K = _width(rng, 128, 11008), _width(rng, 128, 11008)
    most = 10000 * 4096 * 4096 // (N * K)
    M = _log_size(rng, 1, max(1, min(16384, most)))
    case.update(M=M, N=N, K=K)
    if op == "product":
        case.update(back=rng.random() < 0.33, bias=False)
        case["bias"] = not case["back"] and rng.random() < 0.5
        return case
    groups = _log_size(rng, 1, 64)
    while groups * N * K > 32 * 4096 * 2048:
        groups = (groups + 1) // 2
        if groups == 1:
            break
    case.update(groups=groups, skew=rng.choice([0.0, 0.5, 1.0, 2.0]))
    if op == "grouped":
        case["back"] = rng.random() < 0.33
    return case


def _sizes(case):
    """Rows of each group: every row falls to a group at random, group of rank r with weight (r + 1)^-skew."""
    M = case["M"] if "M" in case else case["rows"]
    rng = random.Random(M * 1009 + case["groups"])
    ranks = list(range(case["groups"]))
    rng.shuffle(ranks)
    sizes = [0] * case["groups"]
    for g in rng.choices(range(case["groups"]), weights=[(r + 1.0) ** -case["skew"] for r in ranks], k=M):
        sizes[g] += 1
    return sizes


def _up(n, to):
    return (n + to - 1) // to * to


# ---- the format, by elementary operations --------------------------------------------------------------------------

def _scale_bytes(top, codes):
    """Bytes of the scales from the blocks' largest magnitudes (fp32): the least power of two at which they fit the codes."""
    x, most = TOP[codes]
    m, e = torch.frexp(top)                               # top = m 2^e, 0.5 <= m < 1
    e = e - 1 - x + (m * 2.0 > most / 2.0 ** x).int()
    e = torch.where(top > 0, e, torch.full_like(e, -127))
    return (e.clamp(min=-127) + 127).to(torch.uint8)


def _power(bytes_):
    return torch.ldexp(torch.ones(bytes_.shape, device=bytes_.device), bytes_.int() - 127)


def _blocks(x, rows, cols):
    """[R, C] -> [R / rows, rows, C / cols, cols], zeros where the matrix ends inside a block."""
    R, C = x.shape
    p = torch.nn.functional.pad(x, (0, _up(C, cols) - C, 0, _up(R, rows) - R))
    return p.view(p.shape[0] // rows, rows, p.shape[1] // cols, cols)


def _quantised(x, rows, cols, codes):
    """fp32 [R, C] -> codes [R, C] and scale bytes of its blocks of rows x cols."""
    R, C = x.shape
    b = _blocks(x, rows, cols)
    s = _scale_bytes(b.abs().amax(3).amax(1), codes)
    q = b * (1.0 / _power(s))[:, None, :, None]
    return q.reshape(q.shape[0] * rows, -1)[:R, :C].to(CODES[codes]), s


def _values(q, s, rows, cols):
    """What codes [R, C] stand for, in fp32 (exact)."""
    f = _power(s).repeat_interleave(rows, 0)[:q.shape[0]].repeat_interleave(cols, 1)[:, :q.shape[1]]
    return q.float() * f


def _stored(q, s):
    """Codes with rows a whole number of 128-byte lines apart, scales with rows a multiple of 16 bytes apart."""
    R, C = q.shape
    qs = torch.zeros(R, _up(C, B), dtype=torch.uint8, device=q.device)
    qs[:, :C] = q.view(torch.uint8)
    ss = torch.zeros(s.shape[0], _up(s.shape[1], 16), dtype=torch.uint8, device=q.device)
    ss[:, :s.shape[1]] = s
    return qs.view(q.dtype), ss


def _padded(x, sizes):
    """Rows of groups -> the same with each group filled up to whole blocks by rows of zeros."""
    out = torch.zeros(sum(_up(n, B) for n in sizes), x.shape[1], dtype=x.dtype, device=x.device)
    at = to = 0
    for n in sizes:
        out[to:to + n] = x[at:at + n]
        at, to = at + n, to + _up(n, B)
    return out


# ---- inputs ----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    def activations(rows, cols):
        # a few strong channels, and tokens of different strength
        return normal(rows, cols) * torch.exp(0.8 * normal(cols)) * torch.exp(0.5 * normal(rows))[:, None]

    s = dict(case)
    op, kind = case["op"], case["codes"]
    dt = s["dt"] = TYPES[case["type"]]
    if "groups" in case:
        s["sizes"] = _sizes(case)
        ends = torch.tensor([0] + s["sizes"], dtype=torch.int64).cumsum(0)
        s["offsets"] = ends.to(dev)
    if op in ("rows", "tiles", "columns"):
        rows, K = case["rows"], case["K"]
        source = case.get("from") or rows
        s["x"] = (normal(rows, K) / math.sqrt(K) if op == "tiles" else activations(source, K)).to(dt)
        s["index"] = torch.randint(0, source, (rows,), generator=g, device=dev) if case.get("from") else None
        out_rows = sum(_up(n, B) for n in s["sizes"]) if op == "columns" else rows
        if op == "columns":
            # what a program allocates that knows the number of rows, but not the groups' sizes
            blocks = rows // B + case["groups"]
            s["room"] = (blocks * B, blocks)
            scales = (blocks, _up(K, 16))
        else:
            scales = (rows if op == "rows" else (rows + B - 1) // B, _up((K + B - 1) // B, 16))
        s["q"] = torch.zeros(s["room"][0] if op == "columns" else rows, _up(K, B), dtype=torch.uint8, device=dev).view(CODES[kind])
        s["s"] = torch.zeros(*scales, dtype=torch.uint8, device=dev)
        s["out_rows"] = out_rows
        # a code has four significant bits: 16 bits hold what it stands for
        s["values"] = torch.zeros(s["q"].shape[0], K, dtype=torch.bfloat16, device=dev)
        return s
    M, N, K = case["M"], case["N"], case["K"]
    if op == "wgrad":
        y, x = activations(M, N) * 1e-3, activations(M, K)
        s["a"], s["a_s"] = _stored(*_quantised(_padded(y, s["sizes"]), B, 1, kind))
        s["b"], s["b_s"] = _stored(*_quantised(_padded(x, s["sizes"]), B, 1, "e4m3"))
        s["out"] = torch.empty(case["groups"], N, K, dtype=dt, device=dev)
        return s
    groups = case.get("groups", 1)
    # forward: a [M, K] times b [N, K]; backward: a [M, K], the gradient of K outputs, times b [K, N], the same weights read across
    s["a"], s["a_s"] = _stored(*_quantised(activations(M, K), 1, B, kind))
    shape = (K, N) if case["back"] else (N, K)
    made = [_stored(*_quantised(normal(*shape) / math.sqrt(K), B, B, "e4m3")) for _ in range(groups)]
    s["b"], s["b_s"] = torch.stack([m[0].view(torch.uint8) for m in made]).view(torch.float8_e4m3fn), torch.stack([m[1] for m in made])
    s["bias_v"] = normal(N) * 0.1 if case.get("bias") else None
    s["out"] = torch.empty(M, N, dtype=dt, device=dev)
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------

def _plain(s):
    op, dt, kind = s["op"], s["dt"], s["codes"]
    if op in ("rows", "tiles", "columns"):
        x = s["x"].float()
        if op == "rows" and s["index"] is not None:
            x = x[s["index"]]
        if op == "columns":
            x = _padded(x, s["sizes"])
        block = {"rows": (1, B), "tiles": (B, B), "columns": (B, 1)}[op]
        q, sc = _quantised(x, *block, kind)
        return {"values": _values(q, sc, *block).to(torch.bfloat16), "scale": sc}
    M, N, K = s["M"], s["N"], s["K"]
    if op == "wgrad":
        y = _values(s["a"][:, :N], s["a_s"], B, 1)
        x = _values(s["b"][:, :K], s["b_s"], B, 1)
        out, at = [], 0
        for n in s["sizes"]:
            out.append(torch.matmul(y[at:at + _up(n, B)].t(), x[at:at + _up(n, B)]).to(dt))
            at += _up(n, B)
        return {"out": torch.stack(out)}
    a = _values(s["a"][:, :K], s["a_s"], 1, B)
    out, at = [], 0
    for g, n in enumerate(s["sizes"] if op == "grouped" else [M]):
        if n == 0:
            continue
        w = _values(s["b"][g][:, :N if s["back"] else K], s["b_s"][g], B, B)
        out.append(torch.matmul(a[at:at + n], w if s["back"] else w.t()))
        at += n
    y = torch.cat(out)
    if s["bias_v"] is not None:
        y = y + s["bias_v"]
    return {"out": y.to(dt)}


# ---- the library -------------------------------------------------------------------------------------------------

def _own(s):
    from paper_1609_07061_b200 import binding as q
    op = s["op"]
    if op in ("rows", "tiles", "columns"):
        rows, K = s["rows"], s["K"]
        ldq, lds = s["q"].shape[1], s["s"].shape[1]
        if op == "rows":
            q.qnn_quantize_blocks_f8(s["x"], rows, K, K, s["q"], ldq, s["s"], lds, index=s["index"], src_rows=s["x"].shape[0],
                                     values=s["values"], ld_values=K)
            return {"values": s["values"], "scale": s["s"][:, :(K + B - 1) // B]}
        if op == "tiles":
            q.qnn_quantize_tiles_f8(s["x"], rows, K, K, s["q"], ldq, s["s"], lds, values=s["values"], ld_values=K)
            return {"values": s["values"], "scale": s["s"][:, :(K + B - 1) // B]}
        q.qnn_quantize_columns_f8(s["x"], rows, K, K, s["offsets"], s["groups"], s["q"], ldq, s["s"], lds, values=s["values"], ld_values=K)
        return {"values": s["values"][:s["out_rows"]], "scale": s["s"][:s["out_rows"] // B, :K]}
    M, N, K = s["M"], s["N"], s["K"]
    a, b = s["a"], s["b"]
    if op == "wgrad":
        q.qnn_gemm_f8_wgrad(a, a.shape[1], s["a_s"], s["a_s"].shape[1], b, b.shape[1], s["b_s"], s["b_s"].shape[1], s["offsets"], s["groups"],
                            M, N, K, s["out"], K)
    elif op == "grouped":
        q.qnn_gemm_f8_grouped(a, a.shape[1], s["a_s"], s["a_s"].shape[1], b, b.shape[2], s["b_s"], s["b_s"].shape[2], s["offsets"],
                              s["groups"], M, N, K, s["out"], N, b_transposed=s["back"])
    else:
        q.qnn_gemm_f8(a, a.shape[1], s["a_s"], s["a_s"].shape[1], b[0], b.shape[2], s["b_s"][0], s["b_s"].shape[2], M, N, K, s["out"], N,
                      bias=s["bias_v"], b_transposed=s["back"])
    return {"out": s["out"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    es = 4 if case["type"] == "f32" else 2
    op = case["op"]
    if op in ("rows", "tiles", "columns"):
        rows, K = case["rows"], case["K"]
        source = case.get("from") or rows
        out = sum(_up(n, B) for n in _sizes(case)) if op == "columns" else rows
        block = {"rows": B, "tiles": B * B, "columns": B}[op]
        # the input; codes, what they stand for, and scales; the index or the offsets
        more = 8 * rows if case.get("from") else 8 * (case["groups"] + 1) if op == "columns" else 0
        return {"bytes": min(source, rows) * K * es + out * K * 3 + out * K // block + more, "flops": 3.0 * rows * K}
    M, N, K = case["M"], case["N"], case["K"]
    if op == "wgrad":
        return {"bytes": M * (N + K) + M * (N + K) // B + es * case["groups"] * N * K, "flops": 2.0 * M * N * K}
    used = sum(n > 0 for n in _sizes(case)) if op == "grouped" else 1
    return {"bytes": M * K + M * K // B + used * N * K + es * M * N + (4 * N if case.get("bias") else 0), "flops": 2.0 * M * N * K}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def _doubles(q, s, rows, cols):
    e = s.to(torch.float64) - 127.0
    R, C = q.shape
    r = torch.arange(R, device=q.device) // rows
    c = torch.arange(C, device=q.device) // cols
    return q.to(torch.float64) * torch.exp2(e[r][:, c])


def exact(case, seed):
    s = prepare(case, seed)
    op, f64 = case["op"], torch.float64
    if op in ("rows", "tiles", "columns"):
        x = s["x"].to(f64)
        if op == "rows":
            x = x if s["index"] is None else x.index_select(0, s["index"])
            parts = [x]
        elif op == "columns":
            parts = list(torch.split(x, s["sizes"]))
        else:
            parts = [x]
        low, most = {"e4m3": (-6, 3), "e5m2": (-14, 2)}[case["codes"]], TOP[case["codes"]][1]
        done = []
        for p in parts:
            if p.shape[0] == 0:
                continue
            R, C = p.shape
            if op == "columns":
                p = torch.cat([p, torch.zeros(-R % B, C, dtype=f64, device=p.device)])
            r = torch.arange(p.shape[0], device=p.device) // (1 if op == "rows" else B)
            c = torch.arange(C, device=p.device) // (1 if op == "columns" else B)
            # largest magnitude of every block, by scattering the elements into their blocks
            top = torch.zeros(int(r[-1]) + 1, int(c[-1]) + 1, dtype=f64, device=p.device)
            rowmax = torch.zeros(p.shape[0], top.shape[1], dtype=f64, device=p.device)
            rowmax.scatter_reduce_(1, c.expand_as(p), p.abs(), "amax")
            top.scatter_reduce_(0, r[:, None].expand_as(rowmax), rowmax, "amax")
            step = torch.exp2(torch.ceil(torch.log2(top / most)).clamp(min=-127.0))
            step = torch.where(step * most < top, 2.0 * step, torch.where(step * 0.5 * most >= top, 0.5 * step, step))
            step = step[r][:, c]
            v = p / step
            # spacing of the codes around v
            ulp = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** low[0]))) - low[1])
            done.append((v / ulp).round() * ulp * step)
        return {"values": torch.cat(done), "scale": None}
    M, N, K = case["M"], case["N"], case["K"]
    if op == "wgrad":
        y, x = _doubles(s["a"][:, :N], s["a_s"], B, 1), _doubles(s["b"][:, :K], s["b_s"], B, 1)
        at, out = 0, torch.zeros(case["groups"], N, K, dtype=f64, device=y.device)
        for g, n in enumerate(s["sizes"]):
            out[g] = y[at:at + n].T @ x[at:at + n]
            at += _up(n, B)
        return {"out": out}
    a = _doubles(s["a"][:, :K], s["a_s"], 1, B)
    out = torch.empty(M, N, dtype=f64, device=a.device)
    at = 0
    for g, n in enumerate(s["sizes"] if op == "grouped" else [M]):
        if n:
            w = _doubles(s["b"][g][:, :N if case["back"] else K], s["b_s"][g], B, B)
            torch.matmul(a[at:at + n], w if case["back"] else w.T, out=out[at:at + n])
        at += n
    if s["bias_v"] is not None:
        out += s["bias_v"].to(f64)
    return {"out": out}
