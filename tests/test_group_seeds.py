"""The seeds that an optimiser's groups, of a type each, round their states by."""
import pytest
import torch

import paper_2608_22646_gb300 as cai
from paper_2608_22646_gb300 import train


class Handle:
    def __init__(self, tensors):
        self.tensors = list(tensors)


def test_a_seed_for_every_group(monkeypatch):
    """The first group's is the optimiser's; the same again for a state that is loaded."""
    seeds = []
    monkeypatch.setattr(cai, "cai_adamw_init", lambda tensors, bits: Handle(tensors))
    monkeypatch.setattr(cai, "cai_adamw_step", lambda opt, grads, **kw: seeds.append(kw["seed"]))
    opt = train.AdamW([torch.nn.Parameter(torch.ones(4, dtype=d)) for d in (torch.float32, torch.bfloat16)], seed=5)
    opt.step()
    assert seeds[0] == 5 and seeds[1] != 5
    saved = opt.state_dict()
    opt.seed = 99
    opt.step()
    assert seeds[2] == 99 and seeds[3] not in (99, seeds[1])
    opt.load_state_dict(saved)
    opt.step()
    assert seeds[4:] == seeds[:2] and all(0 <= s < 1 << 32 for s in seeds)


@pytest.mark.gpu
def test_groups_are_rounded_apart():
    """Parameters of two types with the same gradients: of 4096 numbers that lie between two
    codes some are rounded up in one and down in the other.  m / 1.1 of a code is a random
    point between its neighbours: two independent roundings differ for a third of them."""
    n = 4096
    params = [torch.nn.Parameter(torch.zeros(n, dtype=d, device="cuda")) for d in (torch.float32, torch.bfloat16)]
    torch.manual_seed(1)
    g = torch.randn(n, device="cuda").bfloat16()
    for p in params:
        p.grad = g.to(p.dtype)
    with train.AdamW(params, state_bits=8) as opt:
        opt.step()
    a, b = opt.state
    assert torch.equal(a["m_scale"], b["m_scale"])
    for k in "mv":
        share = float((a[k] != b[k]).float().mean())
        assert 0.2 < share < 0.5, share
