"""Sampling, teacher records and distillation on the GPU against 64-bit forms."""
import numpy as np
import pytest
import torch

import paper_2608_22646_gb300 as cai
from tests import logit_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def rows_of(M, V, dtype, seed, grid=None, pad=0, offset=0):
    """[M, V] logits in a buffer whose rows are V + pad apart and start
    `offset` elements in; the bytes around them are NaN."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.randn((M, V), generator=g, device="cuda") * 3.0
    if V > 8:
        z[:, torch.randint(0, V, (3,), generator=g, device="cuda")] += 6.0
    if grid:
        z = torch.round(z / grid) * grid
    buf = torch.full((M * (V + pad) + offset,), float("nan"), dtype=dtype, device="cuda")
    view = buf[offset:].view(M, V + pad)[:, :V]
    view.copy_(z)
    return view


def draw(z, u, **kw):
    M = z.shape[0]
    token = torch.full((M,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((M,), -7.0, device="cuda")
    cai.cai_sample_rows(z, u, token, prob, **kw)
    return token.cpu().numpy(), prob.cpu().numpy()


def per_row(M, x, dtype=F32):
    return None if x is None else torch.as_tensor(np.broadcast_to(x, (M,)).copy()).to(dtype).cuda()


# A weight's relative error: x = (z - max) log2(e) / T is at most 42 in
# magnitude where a weight remains, and carries three roundings (2^-24 each, of
# the scale, the difference and the product) plus exp2's 2 ulp:
# 42 ln 2 * 3 * 2^-24 + 2^-22 < 6e-6.  Shares are quotients of such sums.
REL = 1.2e-5


def check_sampled(z, u, token, prob, T, k, p, min_p):
    """The token's interval of the running sum holds u, its probability is its
    share; rows whose cut lies within rounding of a token's weight are passed
    over.  Returns the number of rows checked."""
    zz = z.double().cpu().numpy()
    uu = u.double().cpu().numpy()
    done = 0
    for r in range(len(uu)):
        ix, share, margin = ref.kept_tokens(zz[r], T[r], int(k[r]), p[r], min_p[r])
        if margin < 10 * REL:
            continue
        done += 1
        at = np.flatnonzero(ix == token[r])
        assert len(at) == 1, (r, token[r])
        cum = np.cumsum(share)
        lo, hi = cum[at[0]] - share[at[0]], cum[at[0]]
        slack = REL + len(zz[r]) * 2.0 ** -41
        assert lo - slack <= uu[r] <= hi + slack, (r, lo, uu[r], hi)
        assert abs(prob[r] - share[at[0]]) <= REL * share[at[0]] + 2.0 ** -40, (r, prob[r], share[at[0]])
    return done


SHAPES = [(1, 1), (3, 2), (2, 63), (5, 1000), (4, 4097), (3, 50003), (1, 126464), (40, 9001)]


@pytest.mark.parametrize("M,V", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("filters", ["none", "topk", "topp", "minp", "all"])
def test_sampled_tokens(M, V, dtype, filters):
    z = rows_of(M, V, dtype, 11 * M + V, pad=M % 3, offset=V % 5)
    rng = np.random.default_rng(V)
    u = torch.rand(M, generator=torch.Generator().manual_seed(V)).cuda()
    T = rng.uniform(0.5, 1.5, M).astype(np.float32)
    k = rng.integers(1, 40, M) if filters in ("topk", "all") else np.zeros(M, int)
    p = rng.uniform(0.3, 0.99, M).astype(np.float32) if filters in ("topp", "all") else np.ones(M, np.float32)
    m = rng.uniform(0.001, 0.05, M).astype(np.float32) if filters in ("minp", "all") else np.zeros(M, np.float32)
    token, prob = draw(z, u, temperature=per_row(M, T), top_k=per_row(M, k, torch.int32),
                       top_p=per_row(M, p), min_p=per_row(M, m))
    done = check_sampled(z, u, token, prob, T, k, p, m)
    assert done >= (M + 1) // 2 or filters != "none"


def test_ties_take_the_lowest_indices():
    """Equal logits: top-k and top-p keep the first of them by index."""
    V = 5001
    z = torch.zeros((4, V), device="cuda")
    z[:, 7::2] = -0.0
    u = torch.tensor([0.0, 0.5, 0.999, 0.25], device="cuda")
    token, prob = draw(z, u, top_k=per_row(4, 10, torch.int32))
    assert token.tolist() == [0, 5, 9, 2] and np.allclose(prob, 0.1, rtol=1e-6)
    token, prob = draw(z, u, top_p=per_row(4, 100.0 / V))
    assert token[0] == 0 and token[2] in (99, 100) and abs(prob[0] - 0.01) < 2e-4
    # Two values: the cut falls inside the upper ones.
    z[:] = -3.0
    z[:, 100:4100:10] = 2.0
    token, _ = draw(z, torch.full((4,), 0.9999, device="cuda"), top_k=per_row(4, [1, 2, 399, 400], torch.int32))
    assert token.tolist() == [100, 110, 100 + 3980, 100 + 3990]


def test_greedy_rows():
    M, V = 6, 12345
    for dtype in (BF16, F32):
        z = rows_of(M, V, dtype, 5, grid=0.5)
        T = per_row(M, [0.0, -1.0, float("nan"), 0.0, 1.0, 0.0])
        token, prob = draw(z, torch.rand(M, device="cuda"), temperature=T,
                           top_k=per_row(M, 3, torch.int32), top_p=per_row(M, 0.1))
        zz = z.double().cpu().numpy()
        for r in (0, 1, 2, 3, 5):
            assert token[r] == zz[r].argmax()
            assert abs(prob[r] - np.exp(zz[r].max() - ref.softmax_lse(zz[r]))) < 1e-5 * prob[r]


@pytest.mark.parametrize("V", [3, 777, 126464])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_without_a_softmax_and_masked_tokens(V, dtype):
    inf = float("inf")
    z = rows_of(8, V, dtype, 3)
    low = torch.finfo(dtype).min
    z[0] = -inf                      # nothing left
    z[1, V // 2] = float("nan")
    z[2, V - 1] = inf
    z[3] = low                       # every token masked with the lowest value: all alike
    z[4] = -inf
    z[4, V - 2] = -5.0               # one token left
    z[5] = low
    z[5, 1] = 0.0
    z[6, :V - 1] = -inf
    u = torch.tensor([0.3, 0.3, 0.3, 0.5, 0.99, 0.99, 0.0, 0.5], device="cuda")
    for kw in ({}, dict(top_k=per_row(8, 2, torch.int32)), dict(top_p=per_row(8, 0.9)),
               dict(temperature=per_row(8, 0.0)), dict(min_p=per_row(8, 0.5))):
        token, prob = draw(z, u, **kw)
        assert np.isnan(prob[:3]).all() and (token[:3] >= 0).all() and (token[:3] < V).all()
        assert token[2] == V - 1
        assert 0 <= token[3] < V and prob[3] > 0
        assert token[4] == V - 2 and prob[4] == 1.0
        assert token[5] == 1 and prob[5] == 1.0
        assert token[6] == V - 1 and prob[6] == 1.0


def test_settings_at_their_ends():
    M, V = 5, 1000
    z = rows_of(M, V, F32, 9)
    top = z.argmax(1).cpu().numpy()
    for kw in (dict(top_k=per_row(M, 1, torch.int32)), dict(top_p=per_row(M, 0.0)),
               dict(top_p=per_row(M, -1.0)), dict(min_p=per_row(M, 1.0)), dict(min_p=per_row(M, 7.0)),
               dict(temperature=per_row(M, 1e-30))):
        token, prob = draw(z, torch.rand(M, device="cuda"), **kw)
        assert (token == top).all() and (prob == 1.0).all(), kw
    # k of V or more, p of 1 or more, min_p of 0: off, the same tokens as none.
    u = torch.rand(M, device="cuda")
    a = draw(z, u)
    b = draw(z, u, temperature=per_row(M, 1.0), top_k=per_row(M, V, torch.int32), top_p=per_row(M, 1.5),
             min_p=per_row(M, 0.0))
    assert (a[0] == b[0]).all() and (a[1] == b[1]).all()
    # u outside [0, 1) is taken as its ends; a temperature of infinity as flat.
    token, _ = draw(z, torch.tensor([-1.0, 0.0, 1.0, 5.0, float("nan")], device="cuda"))
    assert token[0] == 0 and token[1] == 0 and token[4] == 0 and token[2] > V - 200 and token[3] > V - 200
    token, prob = draw(z, torch.full((M,), 0.5, device="cuda"), temperature=per_row(M, float("inf")))
    assert (token == V // 2).all() and np.allclose(prob, 1.0 / V, rtol=1e-6)


def test_the_result_does_not_depend_on_the_batch():
    """The same row gives the same token and probability bits in any batch
    (other batches cut rows over other numbers of CTAs)."""
    V = 70001
    z = rows_of(300, V, BF16, 21)
    u = torch.rand(300, device="cuda")
    kw = dict(temperature=per_row(300, 0.8), top_k=per_row(300, 100, torch.int32), top_p=per_row(300, 0.9))
    token, prob = draw(z, u, **kw)
    for r in (0, 7, 299):
        one = {n: x[r:r + 1] for n, x in kw.items()}
        t1, p1 = draw(z[r:r + 1], u[r:r + 1], **one)
        assert t1[0] == token[r] and p1[0] == prob[r]


def test_offsets_beyond_32_bits():
    ld, V = (1 << 30) + 24, 1003
    buf = torch.zeros((3 * ld,), dtype=BF16, device="cuda")
    z = buf.as_strided((3, V), (ld, 1))
    src = rows_of(3, V, BF16, 2)
    z.copy_(src)
    u = torch.rand(3, device="cuda")
    assert [x.tolist() for x in draw(z, u)] == [x.tolist() for x in draw(src.contiguous(), u)]
    vals, idx, lse = top(z, 5)
    v2, i2, l2 = top(src.contiguous(), 5)
    assert (idx == i2).all() and (vals == v2).all() and (lse == l2).all()
    tv, ti = torch.from_numpy(vals).cuda(), torch.from_numpy(idx).cuda()
    loss, stats = torch.empty(3, device="cuda"), torch.empty((3, 2), device="cuda")
    g2 = torch.empty((3, V), dtype=BF16, device="cuda")
    cai.cai_distill_loss(src, tv, ti, loss, stats, grad=g2, temperature=2.0)
    cai.cai_distill_loss(z, tv, ti, loss, stats, grad=z, temperature=2.0)  # in place, far apart
    assert torch.equal(z, g2)


# ---------------------------------------------------------------- records --

def top(z, K, T=1.0):
    M = z.shape[0]
    v = torch.empty((M, K), device="cuda")
    i = torch.empty((M, K), dtype=torch.int32, device="cuda")
    l = torch.empty(M, device="cuda")
    cai.cai_top_rows(z, v, i, l, temperature=T)
    return v.cpu().numpy(), i.cpu().numpy(), l.cpu().numpy()


@pytest.mark.parametrize("M,V,K", [(1, 1, 1), (3, 5, 5), (2, 64, 7), (4, 513, 512), (5, 4099, 33), (2, 50003, 512),
                                   (1, 152064, 64), (33, 20000, 128), (2, 130, 100)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("grid", [None, 0.5, 100.0])
def test_records(M, V, K, dtype, grid):
    """Values and indices are exact.  lse: each term's relative error is that
    of a sampling weight with the terms that count, at most 6e-6, and the sum's
    rounding is far below; the result is rounded to fp32."""
    z = rows_of(M, V, dtype, V + K, grid=grid, pad=M % 2, offset=K % 3)
    z[0, : V // 3] = -float("inf")
    T = 1.7
    v, i, l = top(z, K, T)
    zz = z.double().cpu().numpy()
    for r in range(M):
        order = ref.order_of(zz[r])[:K]
        assert (i[r] == order).all()
        assert (v[r] == zz[r][order]).all()
        want = ref.softmax_lse(zz[r] / T)
        assert abs(l[r] - want) <= 6e-6 + 2e-7 * abs(want)


def test_records_of_unusual_rows():
    inf, nan = float("inf"), float("nan")
    for dtype in (BF16, F32):
        z = torch.zeros((4, 3000), dtype=dtype, device="cuda")
        z[0] = -inf
        z[1, 10] = nan
        z[1, 20] = inf
        z[1, 30] = 5.0
        z[2, 2999] = inf
        z[3] = torch.finfo(dtype).min
        v, i, l = top(z, 4)
        assert i[0].tolist() == [0, 1, 2, 3] and (v[0] == -inf).all() and l[0] == -inf
        assert i[1].tolist() == [10, 20, 30, 0] and np.isnan(v[1][0]) and v[1][1] == inf and np.isnan(l[1])
        assert i[2].tolist() == [2999, 0, 1, 2] and l[2] == inf
        assert i[3].tolist() == [0, 1, 2, 3] and l[3] == np.float32(torch.finfo(dtype).min)


# ------------------------------------------------------------ distillation --

def teacher_of(z, K, seed, tail, tau):
    M, V = z.shape
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = torch.randn((M, V), generator=g, device="cuda") + torch.nan_to_num(z.float(), neginf=-1e4).clamp(min=-1e4)
    v, i = torch.topk(t, K, 1)
    return v, i.to(torch.int32), torch.logsumexp(t / tau, 1) if tail else None


def loss_of(z, tv, ti, tlse, tau, w, grad=True, out=None):
    M, V = z.shape
    loss = torch.full((M,), -7.0, device="cuda")
    stats = torch.full((M, 2), -7.0, device="cuda")
    g = (torch.full((M, V), 99.0, dtype=z.dtype, device="cuda") if out is None else out) if grad else None
    cai.cai_distill_loss(z, tv, ti, loss, stats, top_lse=tlse, temperature=tau, weight=w, grad=g)
    return loss, stats, g


def check_distill(z, tv, ti, tlse, tau, w, loss, stats, grad, up=None):
    """Against the formulas in 64 bits.  A probability's exponent carries the
    roundings of z log2(e) / tau and of lse, |x| 2^-23 with |x| <= 64 for what
    counts: relative 64 ln 2 * 2^-23 < 6e-6, plus the shared error of lse of the
    same size; a loss is a sum of logarithms with that absolute error.  bf16
    gradients are rounded once more (2^-9 relative).  Tokens of the record
    subtract q from A p: the error is relative to the larger of the two."""
    zz, n = z.double().cpu().numpy(), z.shape[0]
    tvv, tii = tv.double().cpu().numpy(), ti.cpu().numpy()
    for r in range(n):
        wr = 1.0 if w is None else float(w[r])
        L, (a, b), G = ref.distill(zz[r], tvv[r], tii[r], None if tlse is None else float(tlse[r]), tau, wr)
        if up is not None:
            G = G * float(up[r])
        scale = abs(wr) * (1.0 if up is None else abs(float(up[r]))) * tau
        if loss is not None:
            assert abs(float(loss[r]) - L) <= 4e-5 * abs(wr) * tau * tau + 1e-5 * abs(L), (r, float(loss[r]), L)
            assert abs(float(stats[r, 0]) - a) <= 1e-5 + 3e-7 * abs(a)
            if np.isfinite(b):
                assert abs(float(stats[r, 1]) - b) <= 1e-5 + 3e-7 * abs(b)
            else:
                assert float(stats[r, 1]) == b
        if grad is not None:
            got = grad[r].double().cpu().numpy()
            rel = 2.0 ** -8 if z.dtype == BF16 else 2e-5
            given = (tii[r] >= 0) & (tii[r] < len(got))
            size = np.abs(G)
            if scale:
                size[tii[r][given]] += 1e-2 * scale * 1.0 if z.dtype == F32 else 0.0
            tol = rel * size + 2e-6 * scale
            bad = np.abs(got - G) > tol
            assert not bad.any(), (r, np.flatnonzero(bad)[:5], got[bad][:5], G[bad][:5])


@pytest.mark.parametrize("M,V,K", [(1, 2, 1), (3, 40, 5), (4, 1000, 16), (3, 4099, 100), (2, 50003, 64), (1, 126464, 512),
                                   (20, 9001, 33)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [False, True])
def test_distillation(M, V, K, dtype, tail):
    tau = 1.0 if V % 2 else 2.0
    z = rows_of(M, V, dtype, V, pad=M % 3, offset=K % 7)
    tv, ti, tlse = teacher_of(z, K, V + 1, tail, tau)
    if M > 1 and K > 2:
        ti[1, K // 2:] = -1
        ti[1, -1] = V  # beyond the vocabulary: no entry
    w = 0.5 + torch.rand(M, device="cuda")
    if M > 2:
        w[2] = 0.0
    loss, stats, grad = loss_of(z, tv, ti, tlse, tau, w)
    check_distill(z, tv, ti, tlse, tau, w, loss, stats, grad)
    # The loss alone gives the same, and the backward call the upstream multiple.
    l2, s2, _ = loss_of(z, tv, ti, tlse, tau, w, grad=False)
    assert torch.equal(loss, l2) and torch.equal(stats, s2)
    up = torch.rand(M, device="cuda") - 0.3
    g = torch.full((M, V + 3), 99.0, dtype=dtype, device="cuda")[:, 1:V + 1]
    cai.cai_distill_backward(z, tv, ti, stats, up, g, top_lse=tlse, temperature=tau, weight=w)
    check_distill(z, tv, ti, tlse, tau, w, None, None, g, up)
    # In place of the logits (rows as far apart and as aligned as before: the
    # order of the sums follows the address modulo 16).
    z2 = rows_of(M, V, dtype, V, pad=M % 3, offset=K % 7)
    loss_of(z2, tv, ti, tlse, tau, w, out=z2)
    assert torch.equal(z2, grad)


def test_entries_that_name_a_token_twice_add_up():
    z = rows_of(2, 300, F32, 4)
    ti = torch.tensor([[5, 9, 5, 299, 5, 9, 0, -1], [1, 1, 1, 1, 1, 1, 1, 1]], dtype=torch.int32, device="cuda")
    tv = torch.randn((2, 8), device="cuda")
    for tlse in (None, torch.full((2,), 4.0, device="cuda")):
        loss, stats, grad = loss_of(z, tv, ti, tlse, 1.5, None)
        check_distill(z, tv, ti, tlse, 1.5, None, loss, stats, grad)


def test_rows_with_nothing_to_learn_are_not_read():
    z = torch.full((3, 501), float("nan"), device="cuda")
    tv = torch.zeros((3, 4), device="cuda")
    ti = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    ti[0] = 3
    w = torch.tensor([0.0, 1.0, 1.0], device="cuda")
    loss, stats, grad = loss_of(z, tv, ti, None, 1.0, w)
    assert (loss == 0).all() and (stats == 0).all() and (grad == 0).all()
    ti[2, 1] = 7
    loss, stats, grad = loss_of(z, tv, ti, None, 1.0, w)
    assert torch.isnan(loss[2]) and torch.isnan(grad[2]).all() and (grad[:2] == 0).all()


def test_masked_student_logits():
    """Suppressed tokens outside the record have no gradient; a token of the
    record that the student cannot take costs an infinite loss and pulls with
    its whole probability; nothing outside the record: finite gradients."""
    inf = float("inf")
    for dtype in (BF16, F32):
        z = rows_of(3, 999, dtype, 8)
        z[0, 100:200] = -inf
        z[0, 300:310] = torch.finfo(dtype).min
        z[1, 50] = -inf
        ti = torch.tensor([[1, 2, 3], [50, 60, 70], [4, 5, 6]], dtype=torch.int32, device="cuda")
        tv = torch.tensor([[1.0, 2.0, 0.0]] * 3, device="cuda")
        z[2] = -inf
        z[2, 4:7] = 1.0
        tlse = torch.full((3,), 3.0, device="cuda")
        loss, stats, grad = loss_of(z, tv, ti, tlse, 1.0, None)
        check_distill(z[:1], tv[:1], ti[:1], tlse[:1], 1.0, None, loss[:1], stats[:1], grad[:1])
        assert (grad[0, 100:200] == 0).all() and (grad[0, 300:310] == 0).all()
        assert loss[1] == inf and torch.isfinite(grad[1]).all()
        assert abs(float(grad[1, 50]) + np.exp(1.0 - 3.0)) < 1e-3
        assert loss[2] == inf and stats[2, 1] == -inf and torch.isfinite(grad[2]).all()
        assert (grad[2, 7:] == 0).all()


def test_student_far_from_the_rest():
    """The rest's probability is summed, not 1 minus the others: with a record
    that holds all but e^-60 of the student's mass it keeps its digits."""
    z = torch.full((1, 2000), -60.0, device="cuda")
    z[0, 3] = 0.0
    ti = torch.tensor([[3]], dtype=torch.int32, device="cuda")
    tv = torch.tensor([[2.0]], device="cuda")
    tlse = torch.tensor([2.5], device="cuda")
    loss, stats, grad = loss_of(z, tv, ti, tlse, 1.0, None)
    check_distill(z, tv, ti, tlse, 1.0, None, loss, stats, grad)


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(tail):
    """Central differences of the kernel's own loss: with h = 0.05 the
    truncation is h^2 / 6 times a third derivative below tau^-1, 4e-4, and the
    loss's rounding of 2e-6 over 2 h is 2e-5."""
    V, K, tau, h = 37, 6, 1.5, 0.05
    z = rows_of(1, V, F32, 77)
    tv, ti, tlse = teacher_of(z, K, 5, tail, tau)
    _, _, grad = loss_of(z, tv, ti, tlse, tau, None)
    step = torch.eye(V, device="cuda") * h
    many = torch.cat([z + step, z - step])
    n = 2 * V
    loss, _, _ = loss_of(many, tv.expand(n, K).contiguous(), ti.expand(n, K).contiguous(),
                         None if tlse is None else tlse.expand(n).contiguous(), tau, None, grad=False)
    diff = (loss[:V] - loss[V:]) / (2 * h)
    assert (diff - grad[0]).abs().max() < 1e-3


# ------------------------------------------------------ streams, refusals --

def test_other_streams_and_graph_capture():
    z = rows_of(64, 30011, BF16, 13)
    u = torch.rand(64, device="cuda")
    want = draw(z, u, top_p=per_row(64, 0.9))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    token = torch.empty(64, dtype=torch.int32, device="cuda")
    prob = torch.empty(64, device="cuda")
    p = per_row(64, 0.9)
    torch.cuda.synchronize()
    cai.cai_sample_rows(z, u, token, prob, top_p=p, stream=s)
    s.synchronize()
    assert (token.cpu().numpy() == want[0]).all()
    graph = torch.cuda.CUDAGraph()
    token.zero_()
    with torch.cuda.graph(graph):
        cai.cai_sample_rows(z, u, token, prob, top_p=p)
    graph.replay()
    torch.cuda.synchronize()
    assert (token.cpu().numpy() == want[0]).all() and (prob.cpu().numpy() == want[1]).all()


def test_no_rows():
    z = torch.empty((0, 50), device="cuda")
    e = torch.empty(0, device="cuda")
    i = torch.empty(0, dtype=torch.int32, device="cuda")
    cai.cai_sample_rows(z, e, i, e)
    cai.cai_top_rows(z, torch.empty((0, 3), device="cuda"), torch.empty((0, 3), dtype=torch.int32, device="cuda"), e)
    cai.cai_distill_loss(z, torch.empty((0, 3), device="cuda"),
                         torch.empty((0, 3), dtype=torch.int32, device="cuda"), e, torch.empty((0, 2), device="cuda"))


def test_refusals():
    M, V = 2, 100
    z = rows_of(M, V, F32, 1)
    f = torch.zeros(M, device="cuda")
    i = torch.zeros(M, dtype=torch.int32, device="cuda")
    kv, ki = torch.zeros((M, 3), device="cuda"), torch.zeros((M, 3), dtype=torch.int32, device="cuda")
    st = torch.zeros((M, 2), device="cuda")
    for call in (lambda: cai.cai_sample_rows(z.half(), f, i, f), lambda: cai.cai_sample_rows(z.T, f, i, f),
                 lambda: cai.cai_sample_rows(z[:1].expand(2, V), f, i, f),
                 lambda: cai.cai_sample_rows(z.cpu(), f, i, f), lambda: cai.cai_sample_rows(z, f[:1], i, f),
                 lambda: cai.cai_sample_rows(z, f, f, f), lambda: cai.cai_sample_rows(z, f.cpu(), i, f),
                 lambda: cai.cai_sample_rows(z, f, i, f, top_k=f), lambda: cai.cai_top_rows(z, kv, ki[:1], f),
                 lambda: cai.cai_distill_loss(z, kv, ki, f, st, grad=z.bfloat16()),
                 lambda: cai.cai_distill_loss(z, kv, ki, f, f)):
        with pytest.raises(ValueError):
            call()
    wide = torch.zeros((1, 262145), device="cuda")
    many = torch.zeros((M, 101), device="cuda")
    for status, call in (
            (cai.CAI_ERR_SHAPE, lambda: cai.cai_sample_rows(wide, f[:1], i[:1], f[:1])),
            (cai.CAI_ERR_SHAPE, lambda: cai.cai_top_rows(z, many, many.int(), f)),
            (cai.CAI_ERR_ARG, lambda: cai.cai_top_rows(z, kv, ki, f, temperature=0.0)),
            (cai.CAI_ERR_ARG, lambda: cai.cai_top_rows(z, kv, ki, f, temperature=float("inf"))),
            (cai.CAI_ERR_ARG, lambda: cai.cai_distill_loss(z, kv, ki, f, st, temperature=-1.0)),
            (cai.CAI_ERR_ARG, lambda: cai.cai_sample_rows(z, None, i, f)),
            (cai.CAI_ERR_ARG, lambda: cai.cai_distill_backward(z, kv, ki, st, None, z)),
            (cai.CAI_ERR_ARG, lambda: cai.cai_distill_backward(z, kv, ki, st, f, None))):
        with pytest.raises(cai.CaiError) as e:
            call()
        assert e.value.status == status
    # The C entry itself: host memory, a stride below V, a bad dtype.
    L, host = cai.lib(), np.zeros(400, np.float32)
    p = z.data_ptr()
    assert L.cai_sample_rows(host.ctypes.data, 1, V, M, V, 0, 0, 0, 0, f.data_ptr(), i.data_ptr(), f.data_ptr(), 0) == cai.CAI_ERR_ARG
    assert L.cai_sample_rows(p, 1, V - 1, M, V, 0, 0, 0, 0, f.data_ptr(), i.data_ptr(), f.data_ptr(), 0) == cai.CAI_ERR_ARG
    assert L.cai_sample_rows(p, 2, V, M, V, 0, 0, 0, 0, f.data_ptr(), i.data_ptr(), f.data_ptr(), 0) == cai.CAI_ERR_ARG
    assert L.cai_sample_rows(p + 2, 1, V, M, V, 0, 0, 0, 0, f.data_ptr(), i.data_ptr(), f.data_ptr(), 0) == cai.CAI_ERR_ARG
    assert L.cai_sample_rows(p, 1, V, -1, V, 0, 0, 0, 0, f.data_ptr(), i.data_ptr(), f.data_ptr(), 0) == cai.CAI_ERR_SHAPE
    torch.cuda.synchronize()
