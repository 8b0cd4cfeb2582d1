"""Handles of the optimiser are freed by those who made them."""
import pytest
import torch

import paper_2608_22646_gb300 as cai
from paper_2608_22646_gb300 import distill_head, policy_head, train


class Handle:
    def __init__(self, tensors):
        self.tensors = list(tensors)


def test_the_groups_before_a_refused_one(monkeypatch):
    freed = []

    def init(tensors, bits):
        tensors = list(tensors)
        if tensors[0]["param"].dtype == torch.bfloat16:
            raise ValueError("refused")
        return Handle(tensors)

    monkeypatch.setattr(cai, "cai_adamw_init", init)
    monkeypatch.setattr(cai, "cai_adamw_free", freed.append)
    with pytest.raises(ValueError, match="refused"):
        train.AdamW([torch.nn.Parameter(torch.ones(4, dtype=d)) for d in (torch.float32, torch.bfloat16)])
    assert len(freed) == 1


@pytest.mark.gpu
@pytest.mark.parametrize("command,args", [(distill_head, ["--optimiser", "adamw"]),
                                          (distill_head, ["--optimiser", "adamw8", "--norm", "rms"]),
                                          (policy_head, [])])
def test_commands(monkeypatch, capsys, command, args):
    made, init = [], cai.cai_adamw_init
    monkeypatch.setattr(cai, "cai_adamw_init", lambda *a: made.append(init(*a)) or made[-1])
    assert command.main(["--workload", "toy", "--steps", "1"] + args) == 0
    assert made and all(opt.handle == 0 for opt in made)
