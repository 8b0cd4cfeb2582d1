"""The example around the operators on logits, its device calls replaced."""
import types

import pytest
import torch

import paper_2608_22646_gb300 as cai
from paper_2608_22646_gb300 import distill_head

NAN = float("nan")


@pytest.mark.parametrize("probs", [[0.9, 0.1, 0.05, 0.2], [NAN] * 4, [0.2, NAN, 0.1, NAN], [NAN, 0.0, 0.9, 0.3]])
def test_a_block_ends_whatever_its_rows_hold(monkeypatch, probs):
    """Every step keeps a position at least; rows without a softmax come last."""
    P = len(probs)
    kept = []

    def hidden(step):
        assert step <= P, "a step kept nothing"
        return torch.arange(P).float()[:, None].expand(P, 64)

    def logits_of(head, rows, out):
        out[:, 0] = rows[:, 0].to(out.dtype)

    def sample(logits, u, token, prob, **settings):
        token.copy_(logits[:, 0].int())
        prob.copy_(torch.tensor([probs[int(i)] for i in token]))
        kept.append(token.tolist())

    monkeypatch.setattr(cai, "cai_mx4_logits", logits_of)
    monkeypatch.setattr(cai, "cai_sample_rows", sample)
    tokens, steps = distill_head.decode_block(types.SimpleNamespace(V=8), hidden)
    assert tokens.tolist() == list(range(P)) and 1 <= steps <= P
    without = [i for i, p in enumerate(probs) if p != p]
    for masked in kept[:-1]:  # those whose rows have no softmax are masked until the last step
        assert set(without) <= set(masked)
