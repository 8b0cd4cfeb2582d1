"""The preference loss at margins without bounds and between two infinities."""
import math

import pytest
import torch

import paper_2608_22646_gb300 as cai
from paper_2608_22646_gb300 import train

pytestmark = pytest.mark.gpu

INF = float("inf")


def pairs(chosen, rejected, beta, smoothing):
    """(losses, margins, gradients [pairs, 2]) of sequences of one token each."""
    n = len(chosen)
    logp = torch.tensor([chosen, rejected], device="cuda").T.reshape(-1).contiguous()
    cuts = torch.arange(2 * n + 1, dtype=torch.int32, device="cuda")
    loss, margin, grad = (torch.empty(k, device="cuda") for k in (n, n, 2 * n))
    cai.cai_preference_loss(logp, cuts, loss, margin, grad, beta=beta, smoothing=smoothing)
    return loss.tolist(), margin.tolist(), grad.view(n, 2).tolist()


@pytest.mark.parametrize("smoothing", [0.0, 0.0625, 0.5, 1.0])
def test_a_suppressed_token(smoothing):
    """At a margin of -inf the first term, of the share 1 - smoothing, is infinite and the
    second 0; at +inf it is the other way round.  Derivatives by logp: beta times
    smoothing - sigmoid(-margin), which is 1 or 0 there."""
    loss, margin, grad = pairs([-INF, -3.0, -INF], [-2.0, -INF, -INF], 0.5, smoothing)
    assert margin[:2] == [-INF, INF] and math.isnan(margin[2])
    assert loss[0] == (INF if smoothing < 1 else 0.0) and loss[1] == (INF if smoothing else 0.0) and math.isnan(loss[2])
    assert grad[0] == [0.5 * (smoothing - 1), -0.5 * (smoothing - 1)] and grad[1] == [0.5 * smoothing, -0.5 * smoothing]


@pytest.mark.parametrize("smoothing", [0.0, 0.0625, 0.3, 1.0])
def test_finite_margins(smoothing):
    """Of either sign, from 0 to beyond exp's range.  exp is good to 2 ulp and log1p to 1, 2^-22
    and 2^-23 of their term; the share and its product are rounded to 2^-24 of theirs each,
    the sum to 2^-24: less than 2^-21 of the loss."""
    d = [0.0, 1e-6, -1e-6, 0.3, -0.3, 5.0, -5.0, 80.0, -80.0, 1e4, -1e4, 3e38, -3e38]
    loss, margin, _ = pairs(d, [0.0] * len(d), 1.0, smoothing)
    s = float(torch.tensor(smoothing))
    for x, y, m in zip(d, loss, margin):
        x = float(torch.tensor(x))
        share = (1 - s) if x < 0 else s
        want = math.log1p(math.exp(-abs(x))) + share * abs(x)
        assert m == x and abs(y - want) <= 2.0 ** -21 * want, (x, y, want)


def test_a_suppressed_token_through_autograd():
    """Loss +inf, and gradients that are numbers: of the row's softmax and the token."""
    z = torch.zeros((2, 4), device="cuda")
    z[0, 1] = -INF
    z.requires_grad_()
    token = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    logp = train.TokenLogp.apply(z, token, 1.0)
    cuts = torch.arange(3, dtype=torch.int32, device="cuda")
    loss, margin = train.PreferenceLoss.apply(logp, cuts, None, None, 0.5, 0.25)
    loss.sum().backward()
    assert float(loss.detach()) == INF and float(margin) == -INF
    # 0.5 (0.25 - 1) for the chosen row: times [v = t] - p, p = 1/3 beside the token
    want = -0.375 * torch.tensor([-1 / 3, 1.0, -1 / 3, -1 / 3])
    assert torch.allclose(z.grad[0].cpu(), want, rtol=1e-5, atol=0)
    assert torch.allclose(z.grad[1].cpu(), 0.375 * torch.tensor([-0.25, -0.25, 0.75, -0.25]), rtol=1e-5, atol=0)
