"""The operators on logits where they take other paths: many rows (one CTA a
row), flat rows, long top-k lists, rows that are all ties; and the program that
runs all of them together."""
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2608_22646_gb300 as cai
from tests import logit_ref as ref
from tests.test_logit_ops_gpu import (BF16, F32, check_distill, check_sampled, draw, loss_of, per_row, rows_of,
                                      teacher_of, top)

pytestmark = pytest.mark.gpu

MANY = 200  # rows: more than there are SMs


def settings(M, seed):
    """Settings of every kind over the rows: none, top-k, top-p, min-p, all."""
    rng = np.random.default_rng(seed)
    kind = np.arange(M) % 5
    T = rng.uniform(0.5, 1.5, M).astype(np.float32)
    k = np.where((kind == 1) | (kind == 4), rng.integers(1, 300, M), 0)
    p = np.where((kind == 2) | (kind == 4), rng.uniform(0.2, 0.99, M), 1.0).astype(np.float32)
    m = np.where((kind == 3) | (kind == 4), rng.uniform(0.001, 0.1, M), 0.0).astype(np.float32)
    return T, k, p, m


def as_kw(T, k, p, m):
    M = len(T)
    return dict(temperature=per_row(M, T), top_k=per_row(M, k, torch.int32), top_p=per_row(M, p), min_p=per_row(M, m))


@pytest.mark.parametrize("V,dtype,pad", [(40003, BF16, 0), (40003, F32, 5), (65536, BF16, 3), (126464, BF16, 0),
                                         (100001, F32, 0)])
def test_many_rows_sampled(V, dtype, pad):
    z = rows_of(MANY, V, dtype, V, pad=pad, offset=pad)
    z[3] = 0.0                          # all alike
    z[7] *= 0.01                        # nearly flat
    z[11] = torch.randn(V, device="cuda") * 0.5  # a wide nucleus
    z[12] = torch.randn(V, device="cuda") * 0.5
    z[13, 1000:] = -float("inf")
    z[17] = torch.finfo(dtype).min
    z[17, 5] = 1.0
    u = torch.rand(MANY, generator=torch.Generator().manual_seed(V)).cuda()
    T, k, p, m = settings(MANY, V)
    p[[7, 12]], k[[7, 11, 12]] = 0.9, 0
    token, prob = draw(z, u, **as_kw(T, k, p, m))
    done = check_sampled(z, u, token, prob, T, k, p, m)
    assert done >= MANY // 2
    # The same rows few at a time, which clusters of CTAs take.
    for a in (0, 5, 10, 15):
        part = slice(a, a + 5)
        t2, p2 = draw(z[part], u[part], **as_kw(T[part], k[part], p[part], m[part]))
        assert (t2 == token[part]).all() and (p2 == prob[part]).all()


@pytest.mark.parametrize("M", [2, MANY])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_flat_rows_with_a_nucleus(M, dtype):
    """Rows without likely tokens: the cut is found among tens of thousands."""
    V = 50021
    g = torch.Generator(device="cuda")
    g.manual_seed(17)
    z = torch.empty((M, V), dtype=dtype, device="cuda")
    z.copy_(torch.randn((M, V), generator=g, device="cuda") * torch.rand((M, 1), generator=g, device="cuda"))
    u = torch.rand(M, generator=torch.Generator().manual_seed(3)).cuda()
    for share in (0.05, 0.5, 0.97):
        p = np.full(M, share, np.float32)
        one, none = np.ones(M, np.float32), np.zeros(M, np.float32)
        token, prob = draw(z, u, top_p=per_row(M, p))
        # (cuts between ties and within rounding of the share are passed over)
        check_sampled(z, u, token, prob, one, np.zeros(M, int), p, none)
        # Every token drawn is in the kept run of the 64-bit order, or at its edge.
        for r in range(min(M, 8)):
            zz = z[r].double().cpu().numpy()
            order = ref.order_of(zz)
            w = np.exp(zz[order] - zz.max())
            place = int(np.flatnonzero(order == token[r])[0])
            assert (w.cumsum() - w)[place] <= share * w.sum() * (1 + 1e-5) + 1e-5


@pytest.mark.parametrize("M", [1, MANY])
@pytest.mark.parametrize("k", [500, 512, 513, 2500, 39999])
def test_long_top_k(M, k):
    V = 40003
    z = rows_of(M, V, F32, k)
    u = torch.rand(M, generator=torch.Generator().manual_seed(k)).cuda()
    one, none = np.ones(M, np.float32), np.zeros(M, np.float32)
    kk = np.full(M, k)
    token, prob = draw(z, u, top_k=per_row(M, k, torch.int32))
    assert check_sampled(z, u, token, prob, one, kk, one, none) == M
    p = np.full(M, 0.7, np.float32)
    token, prob = draw(z, u, top_k=per_row(M, k, torch.int32), top_p=per_row(M, p))
    check_sampled(z, u, token, prob, one, kk, p, none)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_rows_of_ties(dtype):
    """All logits alike, or two values: first by index, in every path."""
    V = 65539
    z = torch.zeros((MANY, V), dtype=dtype, device="cuda")
    z[1::2] = -4.0
    z[1::2, 3:60003:3] = 1.5
    u = torch.full((MANY,), 0.99999, device="cuda")
    token, prob = draw(z, u, top_k=per_row(MANY, 3000, torch.int32))
    assert (token[0::2] == 2999).all() and (token[1::2] == 3 + 3 * 2999).all()
    assert np.allclose(prob, 1 / 3000, rtol=1e-5)
    token, prob = draw(z, u, top_p=per_row(MANY, 0.25))
    assert (abs(token[0::2] - V // 4) <= 2).all()
    assert (abs(token[1::2] - (3 + 3 * 5000)) < 200).all()  # 20000 heavy tokens, 45539 light
    v, i, l = top(z[:4], 5)
    assert i[0].tolist() == [0, 1, 2, 3, 4] and i[1].tolist() == [3, 6, 9, 12, 15]
    v, i, l = top(z, 300)
    assert (i[0::2] == np.arange(300)).all() and (i[1::2] == 3 + 3 * np.arange(300)).all()


@pytest.mark.parametrize("V,dtype,K,pad", [(40003, BF16, 33, 0), (40003, F32, 512, 5), (126464, BF16, 128, 0),
                                           (100001, F32, 1, 0)])
def test_many_rows_recorded(V, dtype, K, pad):
    z = rows_of(MANY, V, dtype, V + K, pad=pad, offset=pad)
    inf, nan = float("inf"), float("nan")
    z[1] = -inf
    z[2, 77] = nan
    z[3, 5] = inf
    z[4, : V // 2] = -inf
    z[5] = 1.0
    v, i, l = top(z, K, 1.3)
    for r in range(0, MANY, 7):
        zz = z[r].double().cpu().numpy()
        order = ref.order_of(zz)[:K]
        assert (i[r] == order).all() and (v[r] == zz[order]).all()
        want = ref.softmax_lse(zz / 1.3)
        assert abs(l[r] - want) <= 6e-6 + 2e-7 * abs(want)
    assert (v[1] == -inf).all() and (i[1] == np.arange(K)).all() and l[1] == -inf
    assert i[2, 0] == 77 and np.isnan(v[2, 0]) and np.isnan(l[2])
    assert i[3, 0] == 5 and l[3] == inf
    assert (i[5] == np.arange(K)).all()


@pytest.mark.parametrize("V,dtype,K,pad,tail", [(40003, BF16, 33, 0, True), (40003, F32, 100, 5, False),
                                                (126464, BF16, 64, 0, True), (100001, F32, 512, 0, True)])
def test_many_rows_distilled(V, dtype, K, pad, tail):
    z = rows_of(MANY, V, dtype, V + K, pad=pad, offset=pad)
    tv, ti, tlse = teacher_of(z, K, V, tail, 1.5)
    ti[2, K // 2:] = -1
    ti[3] = ti[3, 0].clone()            # one token, named K times
    ti[4] = -1
    w = 0.5 + torch.rand(MANY, device="cuda")
    w[9::10] = 0.0
    loss, stats, grad = loss_of(z, tv, ti, tlse, 1.5, w)
    some = list(range(0, MANY, 9)) + [2, 3, 4, 9]
    pick = lambda x: None if x is None else x[some]  # noqa: E731
    check_distill(z[some], tv[some], ti[some], pick(tlse), 1.5, w[some], loss[some], stats[some], grad[some])
    up = torch.rand(MANY, device="cuda") - 0.3
    g = torch.full((MANY, V + 3), 99.0, dtype=dtype, device="cuda")[:, 1:V + 1]
    cai.cai_distill_backward(z, tv, ti, stats, up, g, top_lse=tlse, temperature=1.5, weight=w)
    check_distill(z[some], tv[some], ti[some], pick(tlse), 1.5, w[some], None, None, g[some], up[some])
    z2 = rows_of(MANY, V, dtype, V + K, pad=pad, offset=pad)
    loss_of(z2, tv, ti, tlse, 1.5, w, out=z2)
    assert torch.equal(z2, grad)


def test_the_operators_together():
    """Records, a 4-bit head trained on them, and a block sampled from it."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-m", "paper_2608_22646_gb300.distill_head", "--steps", "40"], cwd=root,
                         capture_output=True, text=True, timeout=300, check=True).stdout
    said = json.loads(out.strip().splitlines()[-1])
    assert said["loss"][1] < 0.8 * said["loss"][0]
    assert 1 <= said["block_steps"] <= 16 and all(0 <= t < 4096 for t in said["tokens"])


@pytest.mark.parametrize("M", [2, MANY])
@pytest.mark.parametrize("V,dtype,offset", [(262144, BF16, 0), (262143, BF16, 5), (262144, F32, 3), (261000, BF16, 0)])
def test_the_longest_rows_all_alike(M, V, dtype, offset):
    """Every weight is 1, the most that a sum has to hold: the token is the whole
    part of u V and its probability 1 / V, both without rounding."""
    z = rows_of(M, V, dtype, 1, pad=offset, offset=offset)
    z.fill_(0.25)
    u = torch.rand(M, generator=torch.Generator().manual_seed(V)).cuda()
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    want = np.floor(u.cpu().numpy().astype(np.float64) * V)
    for kw in ({}, {"min_p": per_row(M, 0.5)}):
        token, prob = draw(z, u, **kw)
        assert (token == want).all()
        assert (prob == np.float32(1) / np.float32(V)).all()
    token, prob = draw(z, u, temperature=per_row(M, 0.0))
    assert (token == 0).all() and (prob == np.float32(1) / np.float32(V)).all()
    half = draw(z, u, top_p=per_row(M, 0.5))[0]
    assert (half == np.floor(u.cpu().numpy().astype(np.float64) * -(-V // 2))).all()


@pytest.mark.parametrize("temperature", [1e-60, 1e-40, 1e60])
def test_temperatures_beyond_32_bits_are_refused(temperature):
    z = rows_of(2, 100, F32, 1)
    v, i, lse = (torch.empty((2, 4), device="cuda"), torch.empty((2, 4), dtype=torch.int32, device="cuda"),
                 torch.empty(2, device="cuda"))
    with pytest.raises(cai.CaiError):
        cai.cai_top_rows(z, v, i, lse, temperature=temperature)
    loss, stats = torch.empty(2, device="cuda"), torch.empty((2, 2), device="cuda")
    v.zero_(), i.zero_()
    with pytest.raises(cai.CaiError):
        cai.cai_distill_loss(z, v, i, loss, stats, temperature=temperature)


@pytest.mark.parametrize("M", [2, MANY])
@pytest.mark.parametrize("V,K", [(33, 1), (300, 200), (1000, 8), (1000, 256), (2047, 500), (2049, 256), (4000, 512),
                                 (45001, 256)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_records_of_short_rows_and_many_entries(M, V, K, dtype):
    z = rows_of(M, V, dtype, V + K, pad=3, offset=1)
    z[1, V // 2:] = -float("inf")
    v, i, _ = top(z, K)
    zz = z.double().cpu().numpy()
    for r in range(0, M, 7):
        order = ref.order_of(zz[r])[:K]
        assert (i[r] == order).all() and (v[r] == zz[r][order]).all()


@pytest.mark.parametrize("V", [700, 1500, 2048])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_short_rows_sampled(V, dtype):
    z = rows_of(MANY, V, dtype, V, pad=1, offset=3)
    z[4, V // 3:] = -float("inf")
    u = torch.rand(MANY, generator=torch.Generator().manual_seed(V)).cuda()
    T, k, p, m = settings(MANY, V)
    token, prob = draw(z, u, **as_kw(T, k, p, m))
    assert check_sampled(z, u, token, prob, T, k, p, m) >= MANY // 2


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_records_whose_rows_begin_far_below_their_largest(dtype):
    """The first part of a row says little of the rest.  lse: within 6e-6 + 2e-7
    of its size, as for other rows."""
    V, K = 60001, 5
    z = rows_of(MANY, V, dtype, 11, pad=7, offset=1)
    first = 3 * V // 4
    z[0, first + 5] = 30.0
    z[1, first + 6] = 90.0
    z[2, first + 7] = 900.0
    z[3, :first] = -float("inf")
    z[4, :first] = torch.finfo(dtype).min
    z[5] -= 3000.0
    z[6, :first] -= 80.0
    z[7] = torch.finfo(dtype).min
    v, i, l = top(z, K, 1.25)
    zz = z[:16].double().cpu().numpy()
    for r in range(16):
        order = ref.order_of(zz[r])[:K]
        assert (i[r] == order).all() and (v[r] == zz[r][order]).all()
        if r != 7:
            want = ref.softmax_lse(zz[r] / 1.25)
            assert abs(l[r] - want) <= 6e-6 + 2e-7 * abs(want)
    assert abs(l[7] / (zz[7][0] / 1.25) - 1) < 2e-7


@pytest.mark.parametrize("V,dtype", [(152064, F32), (131100, F32), (200003, BF16)])
def test_long_rows_each_to_one_cta(V, dtype):
    """Rows whose kept part is a small share of them."""
    M, K = 160, 200
    z = rows_of(M, V, dtype, V, pad=5, offset=1)
    v, i, _ = top(z, K)
    for r in range(0, M, 23):
        zz = z[r].double().cpu().numpy()
        order = ref.order_of(zz)[:K]
        assert (i[r] == order).all() and (v[r] == zz[order]).all()
    u = torch.rand(M, generator=torch.Generator().manual_seed(V)).cuda()
    T, k, p, m = settings(M, V)
    p[:20], k[:20] = 0.999, 0       # wide nuclei, their weight nearly the whole
    token, prob = draw(z, u, **as_kw(T, k, p, m))
    part = slice(0, 30)
    t2, p2 = draw(z[part], u[part], **as_kw(T[part], k[part], p[part], m[part]))  # by clusters
    assert (t2 == token[part]).all() and (p2 == prob[part]).all()
    assert check_sampled(z[:60], u[:60], token[:60], prob[:60], T[:60], k[:60], p[:60], m[:60]) >= 30
