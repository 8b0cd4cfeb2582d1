"""The 4-bit LM head on the GPU: codes against a 64-bit search among the
values, logits against exact products."""
import numpy as np
import pytest
import torch

import paper_2608_22646_gb300 as cai

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def rounded(x):
    """What blocks of 32 stand for, by search among the midpoints, in 64 bits."""
    b = x.double().reshape(-1, 32)
    high = b.abs().amax(1, keepdim=True)
    powers = torch.tensor([2.0 ** k for k in range(-125, 128)], dtype=torch.float64, device=x.device)
    scale = torch.cat([powers[:1], powers])[torch.bucketize(torch.nan_to_num(high, nan=1.0, posinf=1.0), powers, right=True)] / 4
    y = b.abs() / scale
    values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    middle = (values[1:] + values[:-1]) / 2
    y = torch.nan_to_num(y, nan=0.0, posinf=0.0)
    low, up = torch.bucketize(y, middle), torch.bucketize(y, middle, right=True)
    r = torch.sign(b) * values[torch.where(low % 2 == 0, low, up)] * scale
    bad = ~torch.isfinite(b).all(1, keepdim=True)
    return torch.where(bad, torch.full_like(r, float("nan")), torch.where(high > 0, r, torch.zeros_like(r))).reshape(x.shape)


def values_of(W):
    v = torch.full(W.shape, -7.0, dtype=BF16, device="cuda")
    with cai.cai_mx4_init(W, 1) as head:
        cai.cai_mx4_update(head, W, v)
        torch.cuda.synchronize()
    return v


def same(a, b):
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a.double()), torch.nan_to_num(b))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [0.02, 1.0, 1e-38, 1e-30, 1e30])
@pytest.mark.parametrize("V,H", [(1, 64), (33, 192), (4099, 256)])
def test_values_are_the_nearest(dtype, scale, V, H):
    g = torch.Generator(device="cuda")
    g.manual_seed(V + H)
    W = (torch.randn((V, H), generator=g, device="cuda") * scale).to(dtype)
    W[0, :32] = 0
    assert same(values_of(W), rounded(W))


def test_ties_saturation_and_blocks_without_a_scale():
    W = torch.zeros((8, 64), device="cuda")
    # Every tie, both signs, under a scale of 1 (largest magnitude 4) and of 2^9.
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.2499999, 0.2500001, 7.99, 6.5, 4.0])
    W[0, :12], W[0, 12:24] = ties.cuda(), -ties.cuda()
    W[1] = W[0] * 512.0
    W[2, 5] = float("nan")
    W[3, 40] = float("inf")
    W[4, 3] = -3.4e38
    W[5, 7] = 1e-45
    W[6, :3] = torch.tensor([1e-38, 3e-39, -1.2e-38])
    got = values_of(W)
    assert same(got, rounded(W))
    assert torch.isnan(got[2, :32]).all() and not torch.isnan(got[2, 32:]).any()
    assert got[0, :7].tolist() == [0, 1, 1, 2, 2, 4, 4]
    assert got[0, 9] == 6.0


def product(W, rows, out_dtype, max_rows=None, pad=0, offset=0):
    M, V = rows.shape[0], W.shape[0]
    buf = torch.full((M * (V + pad) + offset + 8,), -7.0, dtype=out_dtype, device="cuda")
    out = buf[offset:offset + M * (V + pad)].view(M, V + pad)[:, :V]
    with cai.cai_mx4_init(W, max_rows or max(1, M)) as head:
        cai.cai_mx4_logits(head, rows, out)
        torch.cuda.synchronize()
        assert cai.cai_mx4_error_bits(head) == 0
    # Nothing outside the rows was written.
    inside = torch.zeros_like(buf, dtype=torch.bool)
    inside[offset:offset + M * (V + pad)].view(M, V + pad)[:, :V] = True
    assert (buf[~inside] == -7.0).all()
    return out


def check(W, rows, out):
    """Products are exact; fp32 sums of H of them err by at most 2^-23 of the
    sum of magnitudes for each step of 64 values and a few inside a step; bf16
    rounds once more (2^-9)."""
    w, x = rounded(W), rounded(rows)
    want, size = x @ w.T, x.abs() @ w.abs().T
    tol = (W.shape[1] / 64 + 8) * 2.0 ** -23 * size
    if out.dtype == BF16:
        tol = tol + 2.0 ** -8 * want.abs()
    err = (out.double() - want).abs()
    assert bool((err <= tol + 1e-300).all()), (err - tol).max()


SHAPES = [(1, 1, 64), (3, 17, 64), (7, 100, 192), (16, 4096, 256), (128, 4096, 256), (129, 333, 320), (300, 5000, 1024),
          (33, 50003, 512), (1, 40000, 4096), (64, 3000, 16384), (257, 153 * 224, 128)]


@pytest.mark.parametrize("M,V,H", SHAPES)
@pytest.mark.parametrize("dtype,out_dtype", [(BF16, BF16), (BF16, F32), (F32, F32)])
def test_logits(M, V, H, dtype, out_dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(M + V + H)
    W = (torch.randn((V, H), generator=g, device="cuda") * 0.02).to(dtype)
    rows = torch.randn((M, H), generator=g, device="cuda")
    rows[:, 3] *= 20.0
    rows = rows.to(dtype)
    check(W, rows, product(W, rows, out_dtype, pad=M % 3, offset=V % 5))
    check(W, rows, product(W, rows, out_dtype, max_rows=M + 200))


def test_rows_and_weights_without_a_scale():
    """A NaN or an infinity spoils its own row or column and nothing else."""
    W = torch.randn((700, 320), device="cuda") * 0.02
    rows = torch.randn((140, 320), device="cuda")
    W[13, 300] = float("inf")
    rows[5, 0] = float("nan")
    rows[139, 200] = float("-inf")
    out = product(W, rows, F32)
    bad = torch.zeros((140, 700), dtype=torch.bool, device="cuda")
    bad[5], bad[139], bad[:, 13] = True, True, True
    assert torch.equal(torch.isnan(out), bad)
    keep_r = [i for i in range(140) if i not in (5, 139)]
    keep_v = [i for i in range(700) if i != 13]
    check(W[keep_v], rows[keep_r], out[keep_r][:, keep_v])


def test_zero_rows_and_zero_weights():
    W = torch.zeros((300, 128), dtype=BF16, device="cuda")
    rows = torch.randn((5, 128), device="cuda").to(BF16)
    assert (product(W, rows, F32) == 0).all()
    W.normal_()
    rows.zero_()
    assert (product(W, rows, F32) == 0).all()


def test_update_many_calls_and_batches():
    """A handle serves calls of any size up to its own in any order, and an
    update replaces the weight."""
    V, H = 2500, 448
    W = torch.randn((V, H), device="cuda") * 0.02
    with cai.cai_mx4_init(W, 400) as head:
        for M in (400, 1, 129, 40, 256, 3):
            rows = torch.randn((M, H), device="cuda")
            out = torch.empty((M, V), device="cuda")
            cai.cai_mx4_logits(head, rows, out)
            check(W, rows, out)
            W = torch.randn((V, H), device="cuda") * 0.5
            cai.cai_mx4_update(head, W)
            cai.cai_mx4_logits(head, rows, out)
            check(W, rows, out)
        cai.cai_mx4_logits(head, rows[:0], out[:0])
        assert cai.cai_mx4_error_bits(head) == 0


def test_other_stream_and_graph():
    V, H, M = 5000, 512, 48
    W = torch.randn((V, H), device="cuda") * 0.02
    rows = torch.randn((M, H), device="cuda")
    out = torch.zeros((M, V), device="cuda")
    with cai.cai_mx4_init(W, M) as head:
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        cai.cai_mx4_logits(head, rows, out, stream=s)
        s.synchronize()
        check(W, rows, out)
        first = out.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cai.cai_mx4_logits(head, rows, out)
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, first)


def test_beyond_32_bits():
    """Logits whose offsets pass 2^31 elements."""
    V, H, M = 300, 64, 3
    W = torch.randn((V, H), device="cuda")
    rows = torch.randn((M, H), device="cuda")
    ld = (1 << 30) + 8
    buf = torch.empty((2 * ld + V,), dtype=BF16, device="cuda")
    out = buf.as_strided((M, V), (ld, 1))
    with cai.cai_mx4_init(W, M) as head:
        cai.cai_mx4_logits(head, rows, out)
        check(W, rows, out)


def test_refusals():
    W = torch.randn((100, 128), device="cuda")
    rows = torch.randn((4, 128), device="cuda")
    out = torch.empty((4, 100), device="cuda")
    for call in (lambda: cai.cai_mx4_init(W.half(), 4), lambda: cai.cai_mx4_init(W.cpu(), 4),
                 lambda: cai.cai_mx4_init(W[:, :64], 4)):
        with pytest.raises(ValueError):
            call()
    for w, n in ((W[:, :32].contiguous(), 4), (W, 0), (W, 65537), (torch.zeros((1, 16448), device="cuda"), 1)):
        with pytest.raises(cai.CaiError) as e:
            cai.cai_mx4_init(w, n)
        assert e.value.status == cai.CAI_ERR_SHAPE
    with cai.cai_mx4_init(W, 4) as head:
        for call in (lambda: cai.cai_mx4_logits(head, rows[:, :64].contiguous(), out),
                     lambda: cai.cai_mx4_logits(head, rows, out[:3]), lambda: cai.cai_mx4_update(head, W[:50]),
                     lambda: cai.cai_mx4_update(head, W, values=W)):
            with pytest.raises(ValueError):
                call()
        with pytest.raises(cai.CaiError) as e:
            cai.cai_mx4_logits(head, torch.zeros((5, 128), device="cuda"), torch.zeros((5, 100), device="cuda"))
        assert e.value.status == cai.CAI_ERR_SHAPE
        L, h = cai.lib(), head.handle
        host = np.zeros(4096, np.float32)
        assert L.cai_mx4_logits(h, host.ctypes.data, 1, 4, out.data_ptr(), 1, 100, 0) == cai.CAI_ERR_ARG
        assert L.cai_mx4_logits(h, rows.data_ptr(), 1, 4, out.data_ptr(), 1, 99, 0) == cai.CAI_ERR_ARG
        assert L.cai_mx4_logits(h, rows.data_ptr() + 4, 1, 3, out.data_ptr(), 1, 100, 0) == cai.CAI_ERR_ARG
        assert L.cai_mx4_logits(h, rows.data_ptr(), 7, 4, out.data_ptr(), 1, 100, 0) == cai.CAI_ERR_ARG
        assert L.cai_mx4_logits(None, rows.data_ptr(), 1, 4, out.data_ptr(), 1, 100, 0) == cai.CAI_ERR_ARG
    assert cai.lib().cai_mx4_init(W.data_ptr(), 1, 100, 128, 4, 0, None) == cai.CAI_ERR_ARG
    # An allocation that fails leaves nothing behind.
    cai.cai_test_fail_alloc_after(2)
    with pytest.raises(cai.CaiError) as e:
        cai.cai_mx4_init(W, 4)
    assert e.value.status == cai.CAI_ERR_NOMEM
    cai.cai_test_fail_alloc_after(0)
