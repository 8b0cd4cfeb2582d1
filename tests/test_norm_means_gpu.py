"""Means of rows: the quotient of the row's sum and its width in every form."""
import pytest
import torch

import paper_2608_22646_gb300 as cai

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("value", [3.0, 1000.0])
@pytest.mark.parametrize("M", [3, 1900])
def test_constant_rows(dtype, value, M):
    """Sums of whole numbers below 2^24 have no rounding, and the quotient is the number itself: the
    mean is exact and y is 0, in calls of many rows and of few, at every width of whole
    vectors from 4104 to 16384."""
    x = torch.full((M * 16384,), value, dtype=dtype, device="cuda")
    y, stats = torch.empty_like(x), torch.empty((M, 2), device="cuda")
    wrong = []
    for H in range(4104, 16385, 8):
        out = y[:M * H].view(M, H)
        cai.cai_norm_rows(x[:M * H].view(M, H), out, stats)
        wrong.append((out != 0).any() | (stats[:, 0] != value).any())
    wrong = torch.stack(wrong).nonzero().flatten() * 8 + 4104
    assert wrong.numel() == 0, (wrong.numel(), wrong[:10].tolist())
