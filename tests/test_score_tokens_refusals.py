"""What examples/score_tokens.py refuses on the host: calls that its buffers could not hold never reach the library."""
import importlib.util
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WIDTH, HIDDEN, VOCAB, TOKENS = 32, 64, 40, 6


@pytest.fixture(scope="module")
def ex():
    import __graft_entry__ as ge
    ge.build()
    spec = importlib.util.spec_from_file_location("score_tokens_on_the_host", os.path.join(ROOT, "examples", "score_tokens.py"))
    m = importlib.util.module_from_spec(spec)
    sys.modules[spec.name] = m
    spec.loader.exec_module(m)
    return m


@pytest.fixture
def calls(ex, monkeypatch):
    """Names of the library's calls that were reached; none of them runs."""
    made = []
    for name in ("qnn_rmsnorm_quant_i8", "qnn_gemm_i8_scaled", "qnn_silu_mul_quant_i8", "qnn_token_logprobs", "qnn_token_logprobs_backward",
                 "qnn_quantize_rows_i8"):
        monkeypatch.setattr(ex.q, name, lambda *a, _n=name, **k: made.append(_n))
    return made


def weights(ex, N, K):
    return ex.Weights8(torch.zeros(N, ex.pitch(K), dtype=torch.int8), torch.ones(N), N, K)


def block(ex, width=WIDTH, hidden=HIDDEN):
    return ex.Block(torch.ones(width), weights(ex, 2 * hidden, width), weights(ex, width, hidden))


def scorer(ex, blocks, max_top=8):
    return ex.Scorer(torch.zeros(VOCAB, WIDTH), blocks, torch.ones(WIDTH), weights(ex, VOCAB, WIDTH), TOKENS, max_top)


def ids(n):
    return torch.zeros(n, dtype=torch.int64)


def test_calls_beyond_the_buffers_are_refused(ex, calls):
    m = scorer(ex, [block(ex)])
    for tokens, targets, top in [(TOKENS, TOKENS, 9), (TOKENS, TOKENS, 20), (2, 2, -1),          # alternatives
                                 (TOKENS + 1, TOKENS + 1, 5), (TOKENS + 1, TOKENS, 0),           # tokens
                                 (TOKENS, TOKENS - 1, 5), (2, TOKENS, 5)]:                       # targets
        with pytest.raises(ValueError):
            m.score(ids(tokens), ids(targets), top)
    with pytest.raises(ValueError):
        scorer(ex, [block(ex)], max_top=VOCAB + 5).score(ids(2), ids(2), VOCAB + 1)
    with pytest.raises(ValueError):
        m.score(ids(3), ids(6)[::2], 2)                                                          # every other element
    g = torch.ones(TOKENS + 1)
    with pytest.raises(ValueError):
        m.logits_gradient(ids(TOKENS + 1), g)
    with pytest.raises(ValueError):
        m.logits_gradient(ids(TOKENS), g[:TOKENS - 1])
    with pytest.raises(ValueError):
        m.logits_gradient(ids(TOKENS), g[:TOKENS], g[:2])
    assert calls == []


def test_calls_within_the_buffers_go_through(ex, calls):
    m = scorer(ex, [block(ex)])
    out = m.score(ids(TOKENS), ids(TOKENS), 8)
    assert out["top_ids"].shape == (TOKENS, 8) and out["logprob"].shape == (TOKENS,)
    assert m.score(ids(2), ids(2), 0)["top_ids"].shape == (2, 0)
    assert m.logits_gradient(ids(2), torch.ones(2)).shape == (2, VOCAB)
    assert calls.count("qnn_token_logprobs") == 2 and calls[-1] == "qnn_token_logprobs_backward"


def test_weights_that_do_not_fit_are_refused(ex, calls):
    for b in (block(ex, hidden=HIDDEN + 32), block(ex, width=WIDTH + 32)):
        with pytest.raises(ValueError):
            scorer(ex, [block(ex), b])
    with pytest.raises(ValueError):
        ex.Scorer(torch.zeros(VOCAB, WIDTH), [], torch.ones(WIDTH), weights(ex, VOCAB, WIDTH + 32), TOKENS)
    with pytest.raises(ValueError):
        ex.Weights8.of(torch.zeros(8, 16).t())
    assert calls == []
    scorer(ex, []).score(ids(1), ids(1), 1)                                                      # no blocks: norm, product, scores
    assert calls == ["qnn_rmsnorm_quant_i8", "qnn_gemm_i8_scaled", "qnn_token_logprobs"]
