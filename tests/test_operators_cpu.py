"""What the operators on logits and the 4-bit head refuse before any device is
asked for, and calls on no rows."""
import pytest
import torch

import paper_2608_22646_gb300 as cai


def test_host_tensors_are_refused_by_the_binding():
    z, f, i = torch.zeros((2, 10)), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: cai.cai_sample_rows(z, f, i, f),
                 lambda: cai.cai_top_rows(z, torch.zeros((2, 3)), torch.zeros((2, 3), dtype=torch.int32), f),
                 lambda: cai.cai_distill_loss(z, torch.zeros((2, 3)), torch.zeros((2, 3), dtype=torch.int32), f,
                                              torch.zeros((2, 2))),
                 lambda: cai.cai_mx4_init(z, 4)):
        with pytest.raises(ValueError):
            call()


def test_sizes_and_types_are_refused_by_the_library():
    L = cai.lib()
    p = 4096  # never read: the sizes are looked at first
    sample = lambda dtype, ld, M, V: L.cai_sample_rows(p, dtype, ld, M, V, 0, 0, 0, 0, p, p, p, 0)  # noqa: E731
    assert sample(cai.CAI_F32, 10, 0, 10) == cai.CAI_OK
    assert sample(2, 10, 1, 10) == cai.CAI_ERR_ARG
    assert sample(cai.CAI_F32, 9, 1, 10) == cai.CAI_ERR_ARG
    assert sample(cai.CAI_F32, 300000, 1, 262145) == cai.CAI_ERR_SHAPE
    assert sample(cai.CAI_F32, 10, -1, 10) == cai.CAI_ERR_SHAPE
    assert sample(cai.CAI_F32, 10, 1, 0) == cai.CAI_ERR_SHAPE
    top = lambda M, V, K, T: L.cai_top_rows(p, cai.CAI_BF16, V, M, V, K, T, p, p, p, 0)  # noqa: E731
    assert top(0, 10, 3, 1.0) == cai.CAI_OK
    for K in (0, 11, -1):
        assert top(1, 10, K, 1.0) == cai.CAI_ERR_SHAPE
    assert top(1, 1000, 513, 1.0) == cai.CAI_ERR_SHAPE
    for T in (0.0, -1.0, float("nan"), float("inf")):
        assert top(1, 10, 3, T) == cai.CAI_ERR_ARG
    h = cai.ctypes.c_void_p()
    init = lambda V, H, n: L.cai_mx4_init(p, cai.CAI_BF16, V, H, n, 0, cai.ctypes.byref(h))  # noqa: E731
    for V, H, n in ((0, 64, 1), (10, 32, 1), (10, 100, 1), (10, 16448, 1), (10, 64, 0), (10, 64, 65537),
                    ((1 << 22) + 1, 64, 1)):
        assert init(V, H, n) == cai.CAI_ERR_SHAPE and not h.value
    assert L.cai_mx4_init(p, 7, 10, 64, 1, 0, cai.ctypes.byref(h)) == cai.CAI_ERR_ARG
    assert L.cai_mx4_init(None, 0, 10, 64, 1, 0, cai.ctypes.byref(h)) == cai.CAI_ERR_ARG
    assert L.cai_mx4_init(p, 0, 10, 64, 1, 0, None) == cai.CAI_ERR_ARG
    assert L.cai_mx4_update(None, p, 0, None, 0) == cai.CAI_ERR_ARG
    assert L.cai_mx4_logits(None, p, 0, 1, p, 0, 10, 0) == cai.CAI_ERR_ARG
    assert L.cai_mx4_error_bits(None, None) == cai.CAI_ERR_ARG
    L.cai_mx4_free(None)
