"""A refused step of the optimiser leaves everything as it was, on the GPU."""
import pytest
import torch

import paper_2608_22646_gb300 as cai
from paper_2608_22646_gb300 import train

pytestmark = pytest.mark.gpu


def made(bits):
    """Two groups: float32 and bf16 parameters."""
    torch.manual_seed(2)
    params = [torch.nn.Parameter(torch.randn(100, device="cuda").to(d)) for d in (torch.float32, torch.bfloat16)]
    for p in params:
        p.grad = torch.randn(100, device="cuda").to(p.dtype)
    return params, train.AdamW(params, lr=1e-2, state_bits=bits)


@pytest.mark.parametrize("bits", [32, 8])
def test_what_is_refused_moves_nothing_and_does_not_count(bits):
    params, opt = made(bits)
    others, plain = made(bits)
    everything = lambda o, ps: [p.detach().clone() for p in ps] + [v.clone() for s in o.state for v in s.values()]  # noqa: E731
    before = everything(opt, params)
    wrong = torch.ones(2, device="cuda")
    for kw, spoil in ((dict(grad_scale=wrong), {}), (dict(lr_step=wrong[:1]), {}), ({}, dict(lr=float("nan"))),
                      ({}, dict(betas=(0.9, 1.0))), ({}, dict(eps=0.0))):
        kept = {k: getattr(opt, k) for k in spoil}
        for k, v in spoil.items():
            setattr(opt, k, v)
        with pytest.raises((ValueError, cai.CaiError)):
            opt.step(**kw)
        for k, v in kept.items():
            setattr(opt, k, v)
        assert opt.steps == 0
    assert all(torch.equal(a, b) for a, b in zip(before, everything(opt, params)))
    opt.step()
    plain.step()
    assert opt.steps == 1
    assert all(torch.equal(a, b) for a, b in zip(everything(opt, params), everything(plain, others)))
    opt.close()
    plain.close()
    with pytest.raises(cai.CaiError):
        opt.step()
    assert opt.steps == 1
