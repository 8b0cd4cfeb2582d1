"""Rows of a CTA that comes late: no row from there on has a number, and nothing hangs."""
import pytest
import torch

import paper_2608_22646_gb300 as cai


def test_refused_before_any_device():
    L, P = cai.lib(), 4096

    def call(M=4, V=4096, ctas=2, late=1, logits=P, grad=P * 5):
        return L.cai_test_late_rows(logits, M, V, P, P, ctas, late, P, P, P, P, grad, None)

    for kw in (dict(M=0), dict(V=2044), dict(V=4098), dict(V=8196), dict(ctas=1), dict(ctas=3), dict(ctas=16), dict(late=-1),
               dict(late=4)):
        assert call(**kw) == cai.CAI_ERR_SHAPE, kw
    assert call(logits=P + 4) == cai.CAI_ERR_ARG and call(grad=P * 5 + 8) == cai.CAI_ERR_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("with_grad", [False, True])
@pytest.mark.parametrize("ctas,V,late", [(2, 5000, 0), (4, 16384, 5), (8, 8192, 39)])
def test_rows_behind_a_late_one(with_grad, ctas, V, late):
    """The row of which a CTA's sums come after the others have given up, and all behind it:
    NaN, every element of the gradient too.  Rows before it are the ordinary call's to the
    rounding of sums that are cut otherwise (2^-20 of an exponential's sum, 2^-19 of its
    logarithm's distance); rows without a token stay 0."""
    M = 40
    g = torch.Generator(device="cuda")
    g.manual_seed(ctas)
    z = torch.randn((M, V), generator=g, device="cuda")
    token = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    token[[3, 20]] = -1
    A = torch.randn(M, generator=g, device="cuda")

    def outputs():
        return [torch.full(s, 7.0, device="cuda") for s in ((M,), (M,), (M, 2), (M,))] + \
            [torch.full((M, V), 7.0, device="cuda") if with_grad else None]

    want, got = outputs(), outputs()
    cai.cai_policy_loss(z, token, A, *want[:4], grad=want[4])
    cai.cai_test_late_rows(z, token, A, *got, ctas=ctas, late_row=late)
    torch.cuda.synchronize()
    row = torch.arange(M, device="cuda")
    idle, gone = token < 0, (row >= late) & (token >= 0)
    for a, b in zip(got, want):
        if a is None:
            continue
        assert torch.isnan(a[gone]).all()
        assert (a[idle] == 0).all()
        rest = ~idle & ~gone
        assert torch.allclose(a[rest], b[rest], rtol=2.0 ** -18, atol=2.0 ** -18)
    again = outputs()  # and the device is as it was
    cai.cai_policy_loss(z, token, A, *again[:4], grad=again[4])
    assert all(torch.equal(a, b) for a, b in zip(again, want) if a is not None)
