"""The next-token example over vocabularies beyond what one dense layer has outputs for, and answers taken in pieces of the batch."""
import numpy as np
import pytest

from paper_2111_08274_amd import next_token
from tests.test_gpu_next_token_blocks import _head

pytestmark = pytest.mark.gpu


def _check_answers(head, x, y, top):
    # as for small vocabularies: 1e-4 is far above what 32-bit sums lose here
    import torch
    logp, entropy, best, top_logp = head.answers(x, y[..., None].contiguous(), top=top)
    p = {k: v.double() for k, v in head.p.items()}
    h = torch.relu(x.double() @ p["w1"] + p["b1"][:, None])
    h = (h - h.mean(-1, keepdim=True)) / torch.sqrt(h.var(-1, unbiased=False, keepdim=True) + 1e-5) * p["gamma"][:, None] + p["beta"][:, None]
    lp = torch.log_softmax(h @ p["w2"] + p["b2"][:, None], -1)
    assert logp.shape == y.shape + (1,) and entropy.shape == y.shape and best.shape == top_logp.shape == y.shape + (top,)
    assert (logp[..., 0] - lp.gather(2, y[..., None].long())[..., 0]).abs().max() < 1e-4
    assert (entropy + (lp.exp() * lp).sum(-1)).abs().max() < 1e-4
    assert (top_logp - lp.topk(top, -1).values).abs().max() < 1e-4 and (lp.gather(2, best.long()) - lp.topk(top, -1).values).abs().max() < 1e-4


@pytest.mark.parametrize("bf16", [0, 1])
def test_rounds_over_a_vocabulary_wider_than_a_layer(bf16):
    import torch
    vocab = (1 << 17) + 3
    out = next_token.run(replicas=2, n_select=1, vocab=vocab, width=16, hidden=32, batch=40, cycles=1, bf16=bf16)
    assert np.isfinite(out["losses"]).all() and bool(torch.isfinite(out["rows"]).all())
    assert -30 < out["answers"]["logp"] < 0 <= out["answers"]["entropy"] <= out["log_vocab"] + 1e-3


def test_answers_over_a_vocabulary_wider_than_a_layer():
    head, x, y = _head(2, 10, 16, 24, 300001)
    _check_answers(head, x, y, 5)


def test_answers_whose_logits_are_formed_a_piece_at_a_time(monkeypatch):
    head, x, y = _head(2, 30, 24, 32, 4001)
    _check_answers(head, x, y, 3)
    whole = head.answers(x, y[..., None].contiguous(), top=3)
    for logits, columns in ((2 * 4001 * 7, 1 << 17), (1, 1000), (2 * 4001 * 30, 8)):      # seven rows, one, all; columns that a piece may have
        monkeypatch.setattr(next_token, "LOGITS", logits)
        monkeypatch.setattr(next_token, "COLUMNS", columns)
        _check_answers(head, x, y, 3)
    monkeypatch.undo()
    assert all(bool((a == b).all()) for a, b in zip(head.answers(x, y[..., None].contiguous(), top=3), whole))


def test_answers_to_no_tokens():
    head, x, y = _head(2, 0, 16, 24, 50)
    assert [tuple(q.shape) for q in head.answers(x, y[..., None].contiguous(), top=2)] == [(2, 0, 1), (2, 0), (2, 0, 2), (2, 0, 2)]
