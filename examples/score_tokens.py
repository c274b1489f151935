"""Scores tokens with a small language model whose layers run on 8-bit integers: the 8-bit calls used together.

The model is a stack of gated feed-forward blocks between an embedding and a vocabulary product (no attention: what is
shown is how norm, products, gate and scores chain).  Weights are quantised once, a scale for each output channel; at run
time no call allocates, so the whole pass may be captured in a CUDA graph.

    python examples/score_tokens.py --tokens 1            one token, as when text is generated
    python examples/score_tokens.py --tokens 512 --grad   a batch, with the gradient of its scores
"""
from __future__ import annotations

import argparse
import os
import sys
from dataclasses import dataclass
from typing import Dict, List, Optional

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1609_07061_b200 import binding as q  # noqa: E402


def pitch(K: int) -> int:
    """Bytes between rows of 8-bit codes: whole 128-byte lines."""
    return q.qnn_tc_row_bytes(K, q.QNN_FORM_I8)


@dataclass
class Weights8:
    """Codes [N, pitch(K)] and channel scales [N] of a weight matrix [N, K]."""
    codes: torch.Tensor
    scale: torch.Tensor
    N: int
    K: int

    @staticmethod
    def of(w: torch.Tensor) -> "Weights8":
        N, K = w.shape
        if w.stride(1) != 1:
            raise ValueError("the elements of a row of the weights must lie next to each other")
        codes = torch.empty(N, pitch(K), dtype=torch.int8, device=w.device)
        scale = torch.empty(N, dtype=torch.float32, device=w.device)
        q.qnn_quantize_rows_i8(w, N, K, w.stride(0), codes, pitch(K), scale)
        return Weights8(codes, scale, N, K)


@dataclass
class Block:
    gamma: torch.Tensor          # [width]
    gate_up: Weights8            # [2 * hidden, width]: gate rows, then up rows
    down: Weights8               # [width, hidden]


class Scorer:
    """Embedding -> blocks of norm, gate/up product, gated activation, down product -> norm -> vocabulary product -> scores."""

    def __init__(self, embedding: torch.Tensor, blocks: List[Block], gamma: torch.Tensor, head: Weights8, max_tokens: int,
                 max_top: int = 8, eps: float = 1e-5):
        self.embedding, self.blocks, self.gamma, self.head, self.eps = embedding, blocks, gamma, head, eps
        self.max_tokens, self.max_top = max_tokens, max_top
        dev, dt, T = embedding.device, embedding.dtype, max_tokens
        self.width, self.hidden, self.vocab = embedding.shape[1], blocks[0].down.K if blocks else 0, head.N
        w, h = self.width, self.hidden
        for i, b in enumerate(blocks):
            if (b.gate_up.N, b.gate_up.K, b.down.N, b.down.K, b.gamma.numel()) != (2 * h, w, w, h, w):
                raise ValueError(f"block {i}: weights of another width or hidden width than {w}, {h}")
        if head.K != w or gamma.numel() != w:
            raise ValueError(f"the last norm or the vocabulary product is not {w} wide")

        def buf(*shape, dtype=dt):
            return torch.empty(*shape, dtype=dtype, device=dev)
        self.x, self.residual = buf(T, self.width), buf(T, self.width)
        self.codes, self.scale = buf(T, pitch(self.width), dtype=torch.int8), buf(T, dtype=torch.float32)
        self.both = buf(T, 2 * self.hidden)
        self.hcodes, self.hscale = buf(T, pitch(self.hidden), dtype=torch.int8), buf(T, dtype=torch.float32)
        self.logits = buf(T, self.vocab)
        self.logprob, self.entropy, self.lse = (buf(T, dtype=torch.float32) for _ in range(3))
        # (flat: the calls write [tokens, top] rows next to each other)
        self.top_logprob, self.top_ids = buf(T * max_top, dtype=torch.float32), buf(T * max_top, dtype=torch.int64)

    def check(self, top: int = 0, **per_token: Optional[torch.Tensor]) -> int:
        """Number of tokens of a call; every argument that the buffers or the calls below could not hold is refused here, on the
        host (the calls take pointers and sizes, and see no buffer's end)."""
        given = {name: t for name, t in per_token.items() if t is not None}
        T = next(iter(given.values())).numel()
        if T > self.max_tokens:
            raise ValueError(f"{T} tokens, but the buffers hold {self.max_tokens}")
        if not 0 <= top <= min(self.max_top, self.vocab):
            raise ValueError(f"{top} alternatives, but the buffers hold {self.max_top} and the vocabulary {self.vocab}")
        for name, t in given.items():
            if t.numel() != T:
                raise ValueError(f"{name} has {t.numel()} elements for {T} tokens")
            if not t.is_contiguous() or t.device != self.embedding.device:
                raise ValueError(f"{name} must be contiguous and on {self.embedding.device}")
        return T

    def norm(self, T: int, gamma: torch.Tensor, first: bool) -> None:
        """residual = x + residual (or x), and its norm as codes."""
        d = self.width
        q.qnn_rmsnorm_quant_i8(self.x, None if first else self.residual, T, d, d, d, gamma, self.eps, self.codes, pitch(d), self.scale,
                               sum_out=self.residual, ld_sum=d)

    def product(self, codes: torch.Tensor, scale: torch.Tensor, w: Weights8, T: int, out: torch.Tensor) -> None:
        q.qnn_gemm_i8_scaled(codes, pitch(w.K), scale, w.codes, pitch(w.K), w.scale, T, w.N, w.K, out, w.N)

    def score(self, tokens: torch.Tensor, targets: torch.Tensor, top: int = 5) -> Dict[str, torch.Tensor]:
        """Log probabilities of `targets`, entropies and the `top` alternatives, one row a token."""
        T, h = self.check(top, tokens=tokens, targets=targets), self.hidden
        torch.index_select(self.embedding, 0, tokens, out=self.x[:T])
        for i, b in enumerate(self.blocks):
            self.norm(T, b.gamma, first=i == 0)
            self.product(self.codes, self.scale, b.gate_up, T, self.both)
            q.qnn_silu_mul_quant_i8(self.both, self.both[:, h:], T, h, 2 * h, 2 * h, self.hcodes, pitch(h), self.hscale)
            self.product(self.hcodes, self.hscale, b.down, T, self.x)
        self.norm(T, self.gamma, first=not self.blocks)
        self.product(self.codes, self.scale, self.head, T, self.logits)
        q.qnn_token_logprobs(self.logits, T, self.vocab, self.vocab, targets, self.logprob, entropy=self.entropy, lse=self.lse, topk=top,
                             top_logprob=self.top_logprob if top else None, top_ids=self.top_ids if top else None)
        return {"logprob": self.logprob[:T], "entropy": self.entropy[:T], "top_logprob": self.top_logprob[:T * top].view(T, top),
                "top_ids": self.top_ids[:T * top].view(T, top)}

    def logits_gradient(self, targets: torch.Tensor, g_logprob: torch.Tensor, g_entropy: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Gradient of the last score() with respect to its logits, written over them."""
        T, V = self.check(targets=targets, g_logprob=g_logprob, g_entropy=g_entropy), self.vocab
        q.qnn_token_logprobs_backward(self.logits, T, V, V, targets, self.lse, self.entropy, g_logprob, g_entropy, self.logits, V)
        return self.logits[:T]


def random_scorer(width: int, hidden: int, vocab: int, blocks: int, max_tokens: int, seed: int = 0, dtype=torch.bfloat16,
                  max_top: int = 8) -> Scorer:
    """A model of random weights of the usual magnitudes."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale
    bs = [Block((1 + 0.1 * normal(width)).to(dtype), Weights8.of(normal(2 * hidden, width, scale=width ** -0.5)),
                Weights8.of(normal(width, hidden, scale=hidden ** -0.5))) for _ in range(blocks)]
    return Scorer(normal(vocab, width).to(dtype), bs, torch.ones(width, dtype=dtype, device="cuda"),
                  Weights8.of(normal(vocab, width, scale=2.0 * width ** -0.5)), max_tokens, max_top)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--top", type=int, default=5)
    ap.add_argument("--grad", action="store_true", help="also the gradient of the mean log probability")
    a = ap.parse_args()
    m = random_scorer(a.width, a.hidden, a.vocab, a.blocks, a.tokens, max_top=a.top)
    ids = torch.randint(0, a.vocab, (a.tokens + 1,), device="cuda")
    tokens, targets = ids[:-1].contiguous(), ids[1:].contiguous()
    runs = 20
    start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    m.score(tokens, targets, a.top)
    start.record()
    for _ in range(runs):
        out = m.score(tokens, targets, a.top)
    stop.record()
    torch.cuda.synchronize()
    print(f"{a.tokens} tokens in {start.elapsed_time(stop) * 1e3 / runs:.0f} us; mean log probability {out['logprob'].mean().item():.3f}, "
          f"mean entropy {out['entropy'].mean().item():.3f}")
    if a.top:
        print("alternatives of the first token:", [(int(i), round(float(p), 3)) for i, p in zip(out["top_ids"][0], out["top_logprob"][0])])
    if a.grad:
        d = m.logits_gradient(targets, torch.full((a.tokens,), 1.0 / a.tokens, device="cuda"))
        print(f"gradient with respect to the logits: norm {d.float().norm().item():.4f}")
    if q.qnn_device_status() != 0:
        raise SystemExit(q.qnn_last_error())


if __name__ == "__main__":
    main()
