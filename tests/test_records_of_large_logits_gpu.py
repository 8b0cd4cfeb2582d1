"""Records of rows whose logits are large all over: the log-sum-exp keeps the
logarithm of how many there are, whatever a product with 1 / T rounds to."""
import numpy as np
import pytest
import torch

from tests import logit_ref as ref
from tests.test_logit_ops_gpu import BF16, F32, rows_of, top

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [4, 200])  # clusters of CTAs, one CTA a row
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1.25, 1.5, 1.7, 2.0, 4.0])
def test_records_of_large_logits(M, dtype, T):
    """lse within 6e-6 + 2e-7 of its size, as for other rows (T in 32 bits is
    what the call takes)."""
    V, K = 60001, 9
    z = rows_of(M, V, dtype, 5, pad=7, offset=1)
    T32 = float(np.float32(T))
    for r, level in enumerate((torch.finfo(dtype).min, -1e30, -1e10, 2.0 ** 33)):
        z[r] = level
    for r, level in ((M - 2, -2.0 ** 32), (M - 1, 3e9)):
        if M > 4:
            z[r] = level
            z[r, 50000:50010] += 2.0 ** 27      # the largest are not in the row's first part
    v, i, l = top(z, K, T)
    for r in {0, 1, 2, 3, M - 2, M - 1}:
        zz = z[r].double().cpu().numpy()
        order = ref.order_of(zz)[:K]
        assert (i[r] == order).all() and (v[r] == zz[order]).all()
        want = ref.softmax_lse(zz / T32)
        assert abs(l[r] - want) <= 6e-6 + 2e-7 * abs(want), (r, l[r], want)
