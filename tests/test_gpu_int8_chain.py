"""The 8-bit calls chained as in examples/score_tokens.py, each stage against the formula on the stage before it in 64 bits.

Every stage takes its inputs as the library left them, so the tolerances are those of a single call: codes within half a
step (plus 3e-3 for what precedes the rounding) of the exact quotient, products within the rounding of bf16 (8 significant
bits: 2^-8) of the exact sum of the codes, scores within (V / 128 + 64) 2^-24 plus four units of the largest logit."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("score_tokens", os.path.join(ROOT, "examples", "score_tokens.py"))
    m = importlib.util.module_from_spec(spec)
    import sys
    sys.modules["score_tokens"] = m
    spec.loader.exec_module(m)
    return m


def codes_match(codes, scale, t64):
    top = t64.abs().amax(1)
    assert ((scale.double() - top / 127).abs() <= 2e-5 * top / 127).all()
    assert (codes[:, :t64.shape[1]].double() - t64 * (127 / top)[:, None]).abs().max().item() <= 0.5 + 3e-3


def product_matches(out, codes, scale, w):
    y = codes[:, :w.K].double() @ w.codes[:, :w.K].double().t() * scale.double()[:, None] * w.scale.double()[None]
    assert ((out.double() - y).abs() <= 2.0 ** -8 * y.abs() + 2.0 ** -23 * y.abs()).all()


def rms(s64, gamma, eps):
    return s64 / torch.sqrt((s64 * s64).mean(1, keepdim=True) + eps) * gamma.double()


@pytest.mark.parametrize("T,width,hidden,vocab", [(1, 256, 512, 4000), (7, 320, 500, 5003), (200, 512, 1024, 8192)])
def test_chain_stage_by_stage(ex, T, width, hidden, vocab):
    m = ex.random_scorer(width, hidden, vocab, 2, T, seed=T)
    ids = torch.randint(0, vocab, (T,), device="cuda")
    targets = torch.randint(0, vocab, (T,), device="cuda")
    x = m.embedding[ids]
    r = None
    for i, b in enumerate(m.blocks):
        m.x[:T] = x
        if r is not None:
            m.residual[:T] = r
        m.norm(T, b.gamma, first=i == 0)
        s = x.float() if i == 0 else x.float() + r.float()
        assert torch.equal(m.residual[:T], s.to(x.dtype))
        codes_match(m.codes, m.scale, rms(s.double(), b.gamma, m.eps))
        m.product(m.codes, m.scale, b.gate_up, T, m.both)
        product_matches(m.both[:T], m.codes, m.scale, b.gate_up)
        ex.q.qnn_silu_mul_quant_i8(m.both, m.both[:, hidden:], T, hidden, 2 * hidden, 2 * hidden, m.hcodes, ex.pitch(hidden), m.hscale)
        g = m.both[:T, :hidden].double()
        codes_match(m.hcodes, m.hscale, g / (1 + torch.exp(-g)) * m.both[:T, hidden:].double())
        m.product(m.hcodes, m.hscale, b.down, T, m.x)
        product_matches(m.x[:T], m.hcodes, m.hscale, b.down)
        x, r = m.x[:T].clone(), m.residual[:T].clone()
    stage = [t.clone() for t in (m.x, m.residual)]
    out = m.score(ids, targets, top=6)                       # the same, as one pass
    assert torch.equal(m.x, stage[0])
    assert torch.equal(m.residual[:T], (stage[0].float() + stage[1].float()).to(x.dtype)[:T])
    codes_match(m.codes, m.scale, rms(x.double() + r.double(), m.gamma, m.eps))
    product_matches(m.logits[:T], m.codes, m.scale, m.head)
    z = m.logits[:T].double()
    logp = torch.log_softmax(z, 1)
    tol = (vocab / 128 + 64) * 2.0 ** -24 + 4 * 2.0 ** -24 * z.abs().amax(1) * 2
    assert ((out["logprob"].double() - logp.gather(1, targets[:, None])[:, 0]).abs() <= tol + 2.0 ** -22 * logp.abs().amax(1)).all()
    assert torch.equal(out["top_ids"], torch.sort(z, dim=1, descending=True, stable=True).indices[:, :6])
    p = logp.exp()
    want = -p / T
    want[torch.arange(T, device="cuda"), targets] += 1.0 / T
    d = m.logits_gradient(targets, torch.full((T,), 1.0 / T, device="cuda"))
    assert ((d.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6 / T).all()
    assert ex.q.qnn_device_status() == 0


def test_one_token_equals_its_row_of_a_batch(ex):
    """A row of a batch of 64 and the same row alone: int32 sums are exact whatever the tiles, and a row's norm is added up in
    the same order (batches of more than two rows an SM use another one)."""
    m = ex.random_scorer(256, 384, 3000, 2, 64, seed=5)
    ids, targets = torch.randint(0, 3000, (64,), device="cuda"), torch.randint(0, 3000, (64,), device="cuda")
    m.score(ids, targets, top=4)
    x, logits = m.x.clone(), m.logits.clone()
    for t in (0, 17, 63):
        m.score(ids[t:t + 1].contiguous(), targets[t:t + 1].contiguous(), top=4)
        assert torch.equal(m.x[0], x[t]) and torch.equal(m.logits[0], logits[t])
