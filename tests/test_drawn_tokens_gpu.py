"""Sampled tokens with nothing passed over: the cut of top-p and the uniform
number lie in the middle of a token's weight, so that the token is known whatever
the weights' rounding; and calls from several threads and streams at once."""
import threading

import numpy as np
import pytest
import torch

import paper_2608_22646_gb300 as cai
from tests import logit_ref as ref
from tests.test_logit_ops_gpu import BF16, F32, REL, draw, per_row, rows_of, top

pytestmark = pytest.mark.gpu


def flat(n, V, dtype, seed):
    """Rows of logits in [-1, 0].  x = (z - max) log2(e) is below 1.45 there: a
    weight is off by three roundings of it and by exp2's 2 ulp, 1.45 ln 2 * 3 *
    2^-24 + 2^-22 < 4.2e-7, a share of the running sum by twice that, u and p by
    2^-25 more: 9e-7.  Half of the least token's share, e^-1 / (2 V (1 - e^-1))
    and 0.29 / V at least, is above that up to V = 300000."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (-torch.rand((n, V), generator=g, device="cuda")).to(dtype)


def middle(cum, at):
    return (cum[at] + (cum[at - 1] if at else 0.0)) / 2


@pytest.mark.parametrize("M", [2, 200])  # clusters of CTAs, one CTA a row
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [1900, 50021, 126464])
@pytest.mark.parametrize("filters", ["none", "topk", "topp", "both"])
def test_flat_rows_draw_the_very_token(M, dtype, V, filters):
    """Cuts from the first token of the order to the last, many thousands among
    them, and in each a token drawn from anywhere in the run."""
    rng = np.random.default_rng(V + M)
    kinds = min(M, 10)
    base = flat(kinds, V, dtype, V)
    zz = base.double().cpu().numpy()
    orders = [ref.order_of(zz[r]) for r in range(kinds)]
    k, p, u = np.zeros(M, int), np.ones(M), np.zeros(M)
    token_of, prob_of = np.zeros(M, int), np.zeros(M)
    for r in range(M):
        order = orders[r % kinds]
        w = np.exp(zz[r % kinds])
        if filters in ("topk", "both"):
            k[r] = int(np.exp(rng.uniform(0, np.log(V - 1))))
        run = order[:k[r]] if k[r] else order
        if filters in ("topp", "both"):
            n = min(len(run), int(np.exp(rng.uniform(0, np.log(len(run) + 1)))))
            cum = np.cumsum(w[run])
            p[r] = middle(cum, n - 1) / cum[-1]
            run = run[:n]
        kept = np.sort(run)
        share = w[kept] / w[kept].sum()
        at = int(rng.integers(len(kept)))
        u[r] = middle(np.cumsum(share), at)
        token_of[r], prob_of[r] = kept[at], share[at]
    z = base[torch.arange(M) % kinds].contiguous()
    token, prob = draw(z, torch.from_numpy(u.astype(np.float32)).cuda(), top_k=per_row(M, k, torch.int32),
                       top_p=per_row(M, p.astype(np.float32)))
    assert (token == token_of).all(), np.flatnonzero(token != token_of)[:5]
    assert (np.abs(prob - prob_of) <= REL * prob_of).all()


@pytest.mark.parametrize("M", [2, 200])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("filters", ["topk", "topp", "minp", "all"])
def test_peaked_rows_draw_the_very_token(M, dtype, filters):
    """Rows with some dozens of likely tokens, every row checked.  Cuts and draws
    are in the middle of shares above 1e-3, forty times a share's rounding (REL) on
    either side; min-p's cut lies between two weights 2e-4 of themselves apart."""
    V, kinds = 40003, 10
    rng = np.random.default_rng(M)
    base = rows_of(kinds, V, dtype, 4)
    at = rng.choice(V, (kinds, 40), replace=False)
    for r in range(kinds):
        base[r, torch.from_numpy(at[r]).cuda()] += torch.from_numpy(12.0 + rng.exponential(1.5, 40)).to(dtype).cuda()
    zz = base.double().cpu().numpy()
    orders = [ref.order_of(zz[r]) for r in range(kinds)]
    k, p, m, u = np.zeros(M, int), np.ones(M), np.zeros(M), np.zeros(M)
    token_of, prob_of = np.zeros(M, int), np.zeros(M)
    for r in range(M):
        order, z = orders[r % kinds], zz[r % kinds]
        w = np.exp(z - z.max())
        run = order
        if filters in ("topk", "all"):
            k[r] = int(rng.integers(5, 40))
            run = run[:k[r]]
        if filters in ("minp", "all"):
            w_run = w[run]
            gaps = np.flatnonzero((w_run[:-1] > 1e-3) & (w_run[1:] < w_run[:-1] * (1 - 2e-4)))
            cut = int(rng.choice(gaps))
            m[r] = (w_run[cut] + w_run[cut + 1]) / 2
            run = run[:cut + 1]
        if filters in ("topp", "all"):
            cum = np.cumsum(w[run])
            n = int(rng.choice(np.flatnonzero(w[run] / cum[-1] > 1e-3)))
            p[r] = middle(cum, n) / cum[-1]
            run = run[:n + 1]
        kept = np.sort(run)
        share = w[kept] / w[kept].sum()
        one = int(rng.choice(np.flatnonzero(share > 1e-3)))
        u[r] = middle(np.cumsum(share), one)
        token_of[r], prob_of[r] = kept[one], share[one]
    z = base[torch.arange(M) % kinds].contiguous()
    token, prob = draw(z, torch.from_numpy(u.astype(np.float32)).cuda(), top_k=per_row(M, k, torch.int32),
                       top_p=per_row(M, p.astype(np.float32)), min_p=per_row(M, m.astype(np.float32)))
    assert (token == token_of).all(), np.flatnonzero(token != token_of)[:5]
    assert (np.abs(prob - prob_of) <= REL * prob_of + 2.0 ** -40).all()


def test_threads_and_streams_at_once():
    """Four threads, each with a stream, rows and outputs of its own: every call
    gives what it gives alone."""
    jobs, wrong = [], []
    for n, (M, V, dtype) in enumerate([(3, 50003, BF16), (40, 9001, F32), (200, 50021, BF16), (1, 126464, F32)]):
        z = rows_of(M, V, dtype, 50 + n)
        u = torch.rand(M, generator=torch.Generator().manual_seed(n)).cuda()
        kw = dict(top_p=per_row(M, 0.9), top_k=per_row(M, 50, torch.int32))
        jobs.append((z, u, kw, draw(z, u, **kw), top(z, 40, 1.5)))
    torch.cuda.synchronize()

    def work(z, u, kw, drawn, recorded):
        M = z.shape[0]
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            token, prob = torch.empty(M, dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
            v, i, l = torch.empty((M, 40), device="cuda"), torch.empty((M, 40), dtype=torch.int32, device="cuda"), torch.empty(M, device="cuda")
            for _ in range(20):
                cai.cai_sample_rows(z, u, token, prob, **kw)
                cai.cai_top_rows(z, v, i, l, temperature=1.5)
                got = [x.cpu().numpy() for x in (token, prob, v, i, l)]
                if not all((a == b).all() for a, b in zip(got, drawn + recorded)):
                    wrong.append((M, z.shape[1]))

    threads = [threading.Thread(target=work, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
