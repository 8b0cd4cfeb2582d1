"""The example's autograd functions on the GPU against their formulas."""
import pytest
import torch

import paper_2608_22646_gb300 as cai
from paper_2608_22646_gb300 import distill_head
from tests.test_mx4_gpu import BF16, F32, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("wanted", ["both", "rows", "W"])
def test_gradients_of_the_4bit_product(dtype, wanted):
    """By W the gradient times the rows, by the rows the gradient times what the
    codes stand for: float32 products of V or M terms, each sum within 2 n 2^-24 of
    the sum of its terms' magnitudes (n at most V = 600, or tf32's 2^-10 where a
    caller allows it, which is not the default); in the rows' type at last."""
    M, V, H = 37, 600, 192
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    W = torch.randn((V, H), generator=g, device="cuda") * 0.02
    rows = torch.randn((M, H), generator=g, device="cuda").to(dtype)
    W.requires_grad_(wanted != "rows")
    rows.requires_grad_(wanted != "W")
    up = torch.randn((M, V), generator=g, device="cuda")
    with cai.cai_mx4_init(W.detach(), M) as head:
        distill_head.Mx4Linear.apply(W, rows, head).backward(up)
        torch.cuda.synchronize()
    u, w, x = up.double(), rounded(W.detach()), rows.detach().double()

    def check(got, a, b, last):
        want, size = a @ b, a.abs() @ b.abs()
        assert got.dtype == last
        tol = 2 * V * 2.0 ** -24 * size + (2.0 ** -8 * want.abs() if last == BF16 else 0.0)
        assert bool(((got.double() - want).abs() <= tol).all())

    if wanted != "rows":
        check(W.grad, u.T, x, F32)
    else:
        assert W.grad is None
    if wanted != "W":
        check(rows.grad, u, w, dtype)
    else:
        assert rows.grad is None
