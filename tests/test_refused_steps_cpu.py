"""Steps of the optimiser that are refused, the library's calls replaced."""
import pytest
import torch

import paper_2608_22646_gb300 as cai
from paper_2608_22646_gb300 import train


class Handle:
    def __init__(self, tensors):
        self.tensors, self.handle = list(tensors), 1


@pytest.fixture
def two_groups(monkeypatch):
    """(optimiser, parameters, calls): a float32 and a bf16 parameter with gradients.  A call
    is refused by what `refuse` has of its handle's place among the groups."""
    calls, refuse = [], {}

    def step(opt, grads, **kw):
        place = [g[2] for g in made.groups].index(opt)
        if place in refuse:
            raise refuse[place]
        calls.append((place, kw))

    monkeypatch.setattr(cai, "cai_adamw_init", lambda tensors, bits: Handle(tensors))
    monkeypatch.setattr(cai, "cai_adamw_step", step)
    monkeypatch.setattr(cai, "cai_adamw_free", lambda opt: setattr(opt, "handle", 0))
    params = [torch.nn.Parameter(torch.ones(40, dtype=d)) for d in (torch.float32, torch.bfloat16)]
    made = train.AdamW(params, seed=5)
    made.refuse = refuse
    for p in params:
        p.grad = torch.ones_like(p)
    return made, params, calls


def test_a_refused_call_is_not_counted(two_groups):
    opt, params, calls = two_groups
    opt.refuse[0] = cai.CaiError.__new__(cai.CaiError)
    versions = [p._version for p in params]
    for _ in range(3):
        with pytest.raises(cai.CaiError):
            opt.step()
    assert opt.steps == 0 and not calls and [p._version for p in params] == versions
    opt.refuse.clear()
    opt.step()
    opt.step()
    assert opt.steps == 2 and [kw["step"] for _, kw in calls] == [1, 1, 2, 2]


@pytest.mark.parametrize("spoil", ["size", "storage", "gradient"])
def test_no_group_moves_where_another_cannot(two_groups, spoil):
    opt, params, calls = two_groups
    held = params[1].data
    if spoil == "size":
        params[1].grad, params[1].data = None, held[:20]
    elif spoil == "storage":
        params[1].data = held.clone()
    else:  # no memory for its dense form, say
        class Parameter:
            dtype, data_ptr, numel = held.dtype, held.data_ptr, held.numel

            @property
            def grad(self):
                raise MemoryError

        opt.groups[1] = ([Parameter()],) + opt.groups[1][1:]
    with pytest.raises((RuntimeError, MemoryError)):
        opt.step()
    assert opt.steps == 0 and not calls
