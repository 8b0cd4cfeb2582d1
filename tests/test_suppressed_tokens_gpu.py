"""Distillation where logits are far from the others: tokens suppressed with the
type's lowest value or another large negative number, in runs that a thread or a
CTA meets first, and rows whose logits are all large."""
import numpy as np
import pytest
import torch

import paper_2608_22646_gb300 as cai
from tests import logit_ref as ref
from tests.test_logit_ops_gpu import BF16, F32, loss_of, rows_of

pytestmark = pytest.mark.gpu

V, K = 50021, 24
FLT_MAX = float(np.finfo(np.float32).max)


def suppressed_rows(M, dtype, tau):
    """Logits of M rows (8 of them unusual), a record of each, and the record's
    log-sum-exp, which leaves about a third of the teacher's mass to the rest."""
    z = rows_of(M, V, dtype, 31, pad=3)
    low = torch.finfo(dtype).min
    g = torch.Generator().manual_seed(7)
    ti = torch.stack([torch.randperm(V // 2, generator=g)[:K] * 2 + 1 for _ in range(M)]).to(torch.int32).cuda()
    tv = torch.randn((M, K), generator=g).cuda()
    z[0, :64] = low                                # what a row's first threads meet first
    for ctas in (1, 2, 4, 8):                      # and a slice's, however the row is cut
        chunk = -(-(-(-V // ctas)) // 64) * 64
        for c in range(ctas):
            z[1, max(0, c * chunk - 24):c * chunk + 40] = low
    z[1, V - 3000:] = low                          # a vocabulary padded with tokens that are none
    z[2, ti[2, :3].long()] = low                   # tokens of the record
    keep = z[3, ti[3].long()].clone()
    z[3] = low                                     # all but the record
    z[3, ti[3].long()] = keep
    z[4, :20000] = -1e30
    z[4, 20000:30000] = -1e10
    z[4, 30000:30100] = low
    z[5] = -1e10                                   # large all over, the likely ones 2^17 above
    z[5, 100:300:7] += 2.0 ** 27
    z[6] = 2.0 ** 33
    z[6, ti[6, :4].long()] += 2.0 ** 28
    z[7] = low                                     # nothing but suppressed tokens
    return z, tv, ti, torch.logsumexp(tv / tau, 1) + 0.4


def softmax_of(z, tau):
    """Shares and the logarithm of their sum relative to the largest, which a sum
    with a number of 10^38 would not show even in 64 bits."""
    e = np.exp((z - z.max()) / tau)
    return e / e.sum(), np.log(e.sum())


def plain(z, tv, ti, tlse, tau, w):
    """(loss, (lse, lse_rest), gradient) of one row in 64 bits."""
    t = tv / tau
    norm = ref.softmax_lse(t) if tlse is None else tlse
    lq = t - norm
    q = np.exp(lq)
    rest = 0.0 if tlse is None else max(0.0, 1.0 - q.sum())
    outside = np.ones(len(z), bool)
    outside[ti] = False
    p, log_all = softmax_of(z, tau)
    p_rest, log_rest = softmax_of(z[outside], tau)  # of the tokens outside among themselves
    kl = (q * (lq - ((z[ti] - z.max()) / tau - log_all))).sum()
    if rest > 0:
        kl += rest * (np.log(rest) - ((z[outside].max() - z.max()) / tau + log_rest - log_all))
    g = (q.sum() + rest) * p
    g[outside] -= rest * p_rest
    g[ti] -= q
    return w * tau * tau * kl, (z.max() / tau + log_all, z[outside].max() / tau + log_rest), w * tau * g


def close(got, want, tol):
    """32 bits cannot hold a loss above their largest number."""
    return got == np.inf if want > FLT_MAX else abs(got - want) <= tol


def check(z, tv, ti, tlse, tau, w, loss, stats, grad, some, up=None):
    """The bounds of the other distillation tests: a probability's exponent carries
    the roundings of the difference from the largest logit and of its product
    with log2(e) / tau, 64 ln 2 * 2^-23 < 6e-6 for what counts; statistics are
    rounded to 32 bits at their size."""
    for r in some:
        wr, ur = float(w[r]), 1.0 if up is None else float(up[r])
        L, (a, b), G = plain(z[r].double().cpu().numpy(), tv[r].double().cpu().numpy(), ti[r].cpu().numpy(),
                             None if tlse is None else float(tlse[r]), tau, wr)
        G = G * ur
        if loss is not None:
            got = float(loss[r])
            assert close(got, L, 4e-5 * abs(wr) * tau * tau + 1e-5 * abs(L)), (r, got, L)
            for got, want in ((float(stats[r, 0]), a), (float(stats[r, 1]), b)):
                assert abs(got - want) <= 1e-5 + 3e-7 * abs(want), (r, got, want)
        scale = abs(wr * ur) * tau
        size = np.abs(G)
        if z.dtype == F32:
            size[ti[r].cpu().numpy()] += 1e-2 * scale
        tol = (2.0 ** -8 if z.dtype == BF16 else 2e-5) * size + 2e-6 * scale
        bad = ~(np.abs(grad[r].double().cpu().numpy() - G) <= tol)  # NaN is bad
        assert not bad.any(), (r, np.flatnonzero(bad)[:5], grad[r].cpu()[bad][:5], G[bad][:5])


@pytest.mark.parametrize("M", [8, 200])  # clusters of CTAs, one CTA a row
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tau", [1.0, 1.5, 2.0, 4.0])
@pytest.mark.parametrize("tail", [False, True])
def test_suppressed_tokens(M, dtype, tau, tail):
    z, tv, ti, tlse = suppressed_rows(M, dtype, tau)
    tlse = tlse if tail else None
    w = (0.5 + torch.rand(M, generator=torch.Generator().manual_seed(1))).cuda()
    some = list(range(8)) + ([M // 2, M - 1] if M > 8 else [])
    loss, stats, grad = loss_of(z, tv, ti, tlse, tau, w)
    check(z, tv, ti, tlse, tau, w, loss, stats, grad, some)
    up = (torch.rand(M, generator=torch.Generator().manual_seed(2)) + 0.3).cuda()
    g = torch.full((M, V), 99.0, dtype=dtype, device="cuda")
    cai.cai_distill_backward(z, tv, ti, stats, up, g, top_lse=tlse, temperature=tau, weight=w)
    check(z, tv, ti, tlse, tau, w, None, None, g, some, up)


@pytest.mark.parametrize("M", [8, 200])
@pytest.mark.parametrize("tail", [False, True])
def test_students_without_a_softmax(M, tail):
    """A NaN or +inf, in the record or not, and rows with nothing above -inf: the
    loss is NaN, and no other row's."""
    inf = float("inf")
    for dtype in (BF16, F32):
        z = rows_of(M, V, dtype, 12)
        ti = torch.arange(K, dtype=torch.int32, device="cuda").mul(3).expand(M, K).contiguous()
        tv = torch.randn((M, K), generator=torch.Generator().manual_seed(4)).cuda()
        tlse = torch.logsumexp(tv, 1) + 0.4 if tail else None
        z[0, 40000] = float("nan")
        z[1, 3] = float("nan")
        z[2, 40000] = inf
        z[3, 3] = inf
        z[4] = -inf
        loss, stats, grad = loss_of(z, tv, ti, tlse, 1.0, None)
        assert torch.isnan(loss[:5]).all() and torch.isfinite(loss[5:]).all()
        assert torch.isfinite(stats[5:]).all() and torch.isfinite(grad[5:].float()).all()
