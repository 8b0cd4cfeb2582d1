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


def quiet(monkeypatch):
    """The library's calls, which leave their outputs at 1."""
    monkeypatch.setattr(cai, "cai_mx4_update", lambda head, W, values=None: None if values is None else values.fill_(1.0))
    monkeypatch.setattr(cai, "cai_mx4_logits", lambda head, rows, out: out.fill_(1.0))
    monkeypatch.setattr(cai, "cai_distill_loss", lambda z, tv, ti, loss, stats, **kw: (loss.fill_(1.0), stats.fill_(1.0)))
    monkeypatch.setattr(cai, "cai_distill_backward", lambda z, tv, ti, stats, up, grad, **kw: grad.fill_(1.0))


def test_a_second_derivative_is_refused(monkeypatch):
    """The gradients are the library's, which autograd cannot go through: an
    error, and not a derivative without them."""
    quiet(monkeypatch)
    z = torch.zeros((2, 5), requires_grad=True)
    record = torch.zeros((2, 3)), torch.zeros((2, 3), dtype=torch.int32), None
    up = torch.ones(2, requires_grad=True)
    (g,) = torch.autograd.grad(distill_head.DistillLoss.apply(z, record, 1.0, None), z, up, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (g * z).sum().backward()
    W, rows = torch.zeros((5, 64), requires_grad=True), torch.zeros((2, 64), requires_grad=True)
    up = torch.ones((2, 5), requires_grad=True)
    g = torch.autograd.grad(distill_head.Mx4Linear.apply(W, rows, None), (W, rows), up, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (g[0].sum() + g[1].sum() + (W * W).sum()).backward()


@pytest.mark.parametrize("which", ["values", "index", "lse", "weight"])
def test_a_change_in_place_between_the_calls_is_noticed(monkeypatch, which):
    """The backward call reads the record and the weights again."""
    quiet(monkeypatch)
    z = torch.zeros((2, 5), requires_grad=True)
    given = dict(values=torch.zeros((2, 3)), index=torch.zeros((2, 3), dtype=torch.int32), lse=torch.zeros(2),
                 weight=torch.ones(2))
    loss = distill_head.DistillLoss.apply(z, (given["values"], given["index"], given["lse"]), 1.0, given["weight"])
    loss.sum().backward(retain_graph=True)
    assert (z.grad == 1.0).all()
    given[which].zero_()
    with pytest.raises(RuntimeError, match="inplace"):
        loss.sum().backward()


def test_what_has_no_gradient_is_refused(monkeypatch):
    quiet(monkeypatch)
    z = torch.zeros((2, 5), requires_grad=True)
    record = torch.zeros((2, 3)), torch.zeros((2, 3), dtype=torch.int32), None
    with pytest.raises(ValueError):
        distill_head.DistillLoss.apply(z, record, 1.0, torch.ones(2, requires_grad=True))
