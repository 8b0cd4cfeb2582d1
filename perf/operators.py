"""Operators on rows of vocabulary logits, and the 4-bit LM head that makes
such rows, as timed cases.

Four things that users of the decoding head do around it:

* sampling tokens at a temperature, with top-k, top-p and min-p per row, from
  given uniform random numbers (`cai_sample_rows`);
* recording a teacher's K largest logits of every row (`cai_top_rows`);
* training a student on those records: the distillation loss and its gradient
  (`cai_distill_loss`, `cai_distill_backward`);
* an LM-head weight kept in microscaled 4-bit floating point (blocks of 32
  E2M1 values under one power-of-two scale): quantising it (`cai_mx4_update`)
  and multiplying quantised rows with it (`cai_mx4_logits`).

Shapes are the repository's workloads (toy, LLaDA, Dream, batched LLaDA, long
Dream) and generic sizes between them.  Logits are a normal bulk with a few
dozen plausible tokens raised above it by exponential amounts, so that rows
range from certain to flat; suppressed tokens sit at -inf or at the type's
lowest value, as a caller's logit processors leave them.
"""
import math

import torch

own = False

LOG2E = 1.4426950408889634
BULK = 2.0       # standard deviation of the bulk of a row's logits
RAISED = 48      # tokens of a row raised above the bulk
SUPPRESSED = 8   # tokens no row may take
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One token for one request: launch and reduction latency.
        dict(name="sample_one_row", op="sample", M=1, V=126464, dtype="bf16", filters="topkp", pad=0),
        # One 64-token block of an odd vocabulary in 32 bits, a nucleus for
        # every row.
        dict(name="sample_block", op="sample", M=64, V=50003, dtype="f32", filters="topp", pad=5),
        # A serving batch: every request with settings of its own, some greedy.
        dict(name="sample_batch", op="sample", M=2048, V=126464, dtype="bf16", filters="mixed", pad=0),
        # A teacher's record of one block.
        dict(name="top_block", op="top", M=32, V=152064, dtype="bf16", K=64, tau=1.0, pad=0),
        # A teacher's record of a training batch, at the distillation's
        # temperature.
        dict(name="top_batch", op="top", M=2000, V=126464, dtype="bf16", K=128, tau=2.0, pad=0),
        # A small model's loss, then its gradient once the caller's own
        # backward pass has reached it.
        dict(name="distill_small", op="distill", M=33, V=4099, dtype="f32", K=16, tau=1.0, tail=False, fused=False, pad=0),
        # A training batch: loss and gradient in one call, the teacher's
        # remaining mass as one class of its own.
        dict(name="distill_batch", op="distill", M=2048, V=126464, dtype="bf16", K=64, tau=2.0, tail=True, fused=True, pad=0),
        # Re-quantising a small model's head from its 32-bit master weights.
        dict(name="quantize_small", op="quantize", V=4096, H=256, dtype="f32"),
        # Re-quantising a full head after a training step.
        dict(name="quantize_head", op="quantize", V=126464, H=4096, dtype="bf16"),
        # The logits of one row: the weight's bytes.
        dict(name="logits_one_row", op="logits", M=1, V=126464, H=4096, out="bf16"),
        # A ragged batch on an odd vocabulary.
        dict(name="logits_ragged", op="logits", M=159, V=50003, H=1024, out="f32"),
        # The serving batch: 2048 rows in the first step of a block.
        dict(name="logits_batch", op="logits", M=2048, V=126464, H=4096, out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["sample", "sample", "top", "distill", "distill", "quantize", "logits", "logits"])
    V = _log_int(rng, 1000, 152064)
    if op in ("sample", "top", "distill"):
        dtype = rng.choice(["bf16", "f32"])
        most = 2000 * 126464 // (2 if dtype == "f32" else 1)  # no more bytes than the listed batches
        M = min(_log_int(rng, 1, 2048), most // V)
        case = dict(op=op, M=M, V=V, dtype=dtype, pad=rng.choice([0, 0, 1, 7, 64]))
        if op == "sample":
            case["filters"] = rng.choice(["none", "topk", "topp", "minp", "topkp", "mixed"])
            return case
        case["K"] = _log_int(rng, 1, 256)
        case["tau"] = rng.choice([1.0, 1.5, 2.0, 4.0])
        if op == "distill":
            case["tail"] = rng.random() < 0.5
            case["fused"] = rng.random() < 0.5
        return case
    H = 64 * _log_int(rng, 4, 64)
    V = min(_log_int(rng, 4096, 152064), 126464 * 4096 // H)
    if op == "quantize":
        return dict(op=op, V=V, H=H, dtype=rng.choice(["bf16", "f32"]))
    return dict(op=op, M=_log_int(rng, 1, 2048), V=V, H=H, out=rng.choice(["bf16", "f32"]))


# ------------------------------------------------------------------ inputs --

def _generator(seed, of=0):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 16 + of) & ((1 << 62) - 1))
    return g


def _logits(case, g):
    """[M, V] logits, a view of rows `pad` elements longer."""
    M, V, dtype = case["M"], case["V"], DTYPES[case["dtype"]]
    z = torch.randn((M, V), generator=g, device="cuda").mul_(BULK)
    # One raised token in each of RAISED equal parts of the vocabulary.
    part = torch.arange(RAISED, device="cuda") + torch.rand((M, RAISED), generator=g, device="cuda")
    at = (part * (V / RAISED)).to(torch.int64).clamp_(max=V - 1)
    lift = torch.empty((M, RAISED), device="cuda").exponential_(0.3, generator=g)
    z.scatter_add_(1, at, lift + 6.0)
    z[:, torch.randint(0, V, (SUPPRESSED,), generator=g, device="cuda")] = (
        -math.inf if case["dtype"] == "bf16" else torch.finfo(dtype).min)
    buf = torch.full((M, V + case["pad"]), math.nan, dtype=dtype, device="cuda")
    buf[:, :V] = z
    return buf[:, :V]


def _settings(case, g):
    """Temperature, top-k, top-p and min-p of every row."""
    M, kind = case["M"], case["filters"]

    def uniform(lo, hi):
        return lo + (hi - lo) * torch.rand(M, generator=g, device="cuda")

    def some(p):
        return torch.rand(M, generator=g, device="cuda") < p

    t = uniform(0.6, 1.2)
    k = torch.zeros(M, dtype=torch.int32, device="cuda")
    p = torch.ones(M, device="cuda")
    m = torch.zeros(M, device="cuda")
    k_draw = torch.exp(uniform(math.log(5.0), math.log(200.0))).to(torch.int32)
    p_draw, m_draw = uniform(0.8, 0.98), uniform(0.01, 0.1)
    if kind in ("topk", "topkp"):
        k = k_draw
    if kind in ("topp", "topkp"):
        p = p_draw
    if kind == "minp":
        m = m_draw
    if kind == "mixed":
        k = torch.where(some(0.5), k_draw, k)
        p = torch.where(some(0.5), p_draw, p)
        m = torch.where(some(0.25), m_draw, m)
        t = torch.where(some(0.125), torch.zeros_like(t), t)
    return t, k, p, m


def _teacher(case, z, g):
    """A teacher near the student: its K largest logits per row, where they
    are, and its log-sum-exp at the distillation's temperature."""
    M, K = case["M"], min(case["K"], case["V"])
    t = torch.randn(z.shape, generator=g, device="cuda").mul_(0.8)
    t.add_(torch.nan_to_num(z.float(), neginf=-1e4).clamp_(min=-1e4), alpha=0.9)
    values, index = torch.topk(t, K, dim=1)
    lse = torch.logsumexp(t / case["tau"], 1) if case["tail"] else None
    index = index.to(torch.int32)
    # A tenth of the rows have a record that is only partly filled.
    short = torch.rand((M, 1), generator=g, device="cuda") < 0.1
    index[short & (torch.arange(K, device="cuda") >= max(1, K // 2))[None]] = -1
    return values, index, lse


def _row_weights(case, g):
    """Each row's share of the loss: positions that are not masked have none,
    one in eight here."""
    w = 0.5 + torch.rand(case["M"], generator=g, device="cuda")
    w[7::8] = 0.0
    return w / case["M"]


def _weight(V, H, dtype, g):
    W = torch.empty((V, H), dtype=dtype, device="cuda")
    for r in range(0, V, 16384):
        n = min(16384, V - r)
        W[r:r + n] = torch.randn((n, H), generator=g, device="cuda") * 0.02
    return W


def _inputs(case, seed):
    """What both sides are given, from the seed alone."""
    op, st = case["op"], {}
    if op in ("sample", "top", "distill"):
        st["logits"] = z = _logits(case, _generator(seed, 0))
        g = _generator(seed, 1)
        if op == "sample":
            st["t"], st["k"], st["p"], st["m"] = _settings(case, g)
            st["u"] = torch.rand(case["M"], generator=g, device="cuda")
        elif op == "distill":
            st["values"], st["index"], st["lse"] = _teacher(case, z, g)
            st["weight"] = _row_weights(case, g)
            st["upstream"] = 0.5 + torch.rand(case["M"], generator=g, device="cuda")
        return st
    dtype = DTYPES[case["dtype"]] if op == "quantize" else torch.bfloat16
    st["W"] = _weight(case["V"], case["H"], dtype, _generator(seed, 2))
    if op == "logits":
        g = _generator(seed, 3)
        # Normalised hidden states with a few channels far above the others.
        x = torch.randn((case["M"], case["H"]), generator=g, device="cuda")
        x[:, torch.randint(0, case["H"], (3,), generator=g, device="cuda")] *= 12.0
        st["rows"] = x.to(torch.bfloat16)
    return st


class _Mx4:
    """Owns a 4-bit head's handle."""

    def __init__(self, cai, W, max_rows):
        self.cai, self.handle = cai, cai.cai_mx4_init(W, max_rows)

    def __del__(self):
        self.cai.cai_mx4_free(self.handle)


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"], op = case, case["op"]
    if not own:
        if op == "logits":
            st["W4"] = _rounded(st.pop("W").float())  # the weight laid out once, as the handle below
        return st
    import paper_2608_22646_gb300 as cai
    st["cai"] = cai

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if op == "sample":
        st["token"], st["prob"] = empty(case["M"], torch.int32), empty(case["M"], torch.float32)
    elif op == "top":
        K = min(case["K"], case["V"])
        st["values"], st["index"] = empty((case["M"], K), torch.float32), empty((case["M"], K), torch.int32)
        st["lse"] = empty(case["M"], torch.float32)
    elif op == "distill":
        st["loss"], st["stats"] = empty(case["M"], torch.float32), empty((case["M"], 2), torch.float32)
        st["grad"] = empty((case["M"], case["V"]), DTYPES[case["dtype"]])
    elif op == "quantize":
        st["head"] = _Mx4(cai, st["W"], 1)
        st["rounded"] = empty((case["V"], case["H"]), torch.bfloat16)
    else:
        st["head"] = _Mx4(cai, st.pop("W"), case["M"])
        st["out"] = empty((case["M"], case["V"]), DTYPES[case["out"]])
    return st


# ------------------------------------------------------------- plain forms --

def _plain_sample(st):
    """Tokens are ordered by falling logit, ties by index.  A token's weight is
    2^((z - max z) log2(e) / T) in units of 2^-40, rounded to a whole number, so
    that sums do not depend on their order.  Top-k and min-p keep what they
    name; top-p keeps the shortest run of what is left that holds a share p of
    its weight; the token is the first, by index, where the running weight
    passes u times the whole."""
    z = st["logits"].float()
    t, k, p, m, u = (st[n][:, None] for n in "tkpmu")
    V = z.shape[1]
    greedy = t == 0
    top = z.amax(1, keepdim=True)
    scale = torch.full_like(t, LOG2E) / torch.where(greedy, torch.ones_like(t), t)
    order, index = torch.sort(z, dim=1, descending=True, stable=True)
    e = torch.exp2((order - top) * scale)
    w = torch.round(e * 2.0 ** 40).to(torch.int64)
    whole = w.sum(1, keepdim=True)
    place = torch.arange(V, device=z.device)[None]
    k = torch.where(greedy, torch.ones_like(k), torch.where(k <= 0, torch.full_like(k, V), k))
    w = torch.where((place < k) & (e >= m.clamp(max=1.0)), w, torch.zeros_like(w))
    del e, order
    target = torch.ceil(p.double() * w.sum(1, keepdim=True).double()).to(torch.int64).clamp(min=1)
    w = torch.where((p >= 1.0) | (w.cumsum(1) - w < target), w, torch.zeros_like(w))
    w = torch.zeros_like(w).scatter_(1, index, w)
    del index
    left = w.sum(1, keepdim=True)
    drawn = torch.minimum((u.double() * left.double()).to(torch.int64), left - 1)
    token = (w.cumsum(1) <= drawn).sum(1, keepdim=True)
    prob = w.gather(1, token).double() / torch.where(greedy, whole, left).double()
    return dict(token=token[:, 0].to(torch.int32), prob=prob[:, 0].float())


def _plain_top(st):
    case, z = st["case"], st["logits"].float()
    K = min(case["K"], case["V"])
    top = z.amax(1, keepdim=True)
    lse = top / case["tau"] + torch.log(torch.exp((z - top) / case["tau"]).sum(1, keepdim=True))
    order, index = torch.sort(z, dim=1, descending=True, stable=True)
    return dict(values=order[:, :K].contiguous(), index=index[:, :K].to(torch.int32), lse=lse[:, 0])


def _plain_distill(st):
    """q: the teacher's probabilities of its K tokens, renormalised over them
    or, with its log-sum-exp given, as they are, the rest being one class.
    Loss: w tau^2 sum_c q_c (log q_c - log p_c) over the classes."""
    case, tau = st["case"], st["case"]["tau"]
    x = st["logits"].float() / tau
    M, V = x.shape
    index, t = st["index"].long(), st["values"] / tau
    given = index >= 0
    at = index.clamp(min=0)
    inside = torch.zeros((M, V + 1), dtype=torch.bool, device=x.device)
    inside = inside.scatter_(1, torch.where(given, at, torch.full_like(at, V)), True)[:, :V]
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    others = torch.where(inside, torch.zeros_like(e), e).sum(1, keepdim=True)
    lse, lse_rest = top + torch.log(total), top + torch.log(others)
    zero = torch.zeros_like(t)
    if case["tail"]:
        q = torch.where(given, torch.exp(t - st["lse"][:, None]), zero)
        rest = (1.0 - q.sum(1, keepdim=True)).clamp(min=0.0)
    else:
        high = torch.where(given, t, torch.full_like(t, -math.inf)).amax(1, keepdim=True)
        q = torch.where(given, torch.exp(t - high), zero)
        q = q / q.sum(1, keepdim=True)
        rest = torch.zeros_like(top)
    logp = x.gather(1, at) - lse
    kl = torch.where(q > 0, q * (torch.log(q) - logp), zero).sum(1, keepdim=True)
    kl = kl + torch.where(rest > 0, rest * (torch.log(rest) - (lse_rest - lse)), torch.zeros_like(rest))
    w = st["weight"][:, None]
    loss = w * (tau * tau) * kl
    up = w if case["fused"] else w * st["upstream"][:, None]
    whole = q.sum(1, keepdim=True) + rest
    prob = e / total
    share = torch.where(rest > 0, rest * total / others, torch.zeros_like(rest))
    grad = prob * torch.where(inside, whole, whole - share)
    hit = torch.zeros((M, V + 1), device=x.device)
    hit.scatter_add_(1, torch.where(given, at, torch.full_like(at, V)), q)
    grad = (up * tau) * (grad - hit[:, :V])
    live = (w != 0) & given.any(1, keepdim=True)
    none = torch.zeros_like(lse)
    stats = torch.cat([torch.where(live, lse, none), torch.where(live, lse_rest, none)], 1)
    return dict(loss=torch.where(live, loss, none)[:, 0], stats=stats,
                grad=torch.where(live, grad, torch.zeros_like(grad)).to(st["logits"].dtype))


def _rounded(x):
    """The values that blocks of 32 stand for in microscaled E2M1: the scale is
    2^(floor(log2 max|x|) - 2), elements go to the nearest of 0, 0.5, 1, 1.5,
    2, 3, 4, 6 (ties to the even code), larger ones to 6."""
    shape = x.shape
    x = x.reshape(-1, 32)
    high = x.abs().amax(1, keepdim=True)
    power = (torch.frexp(high)[1] - 3).clamp(min=-127)
    power = torch.where(high > 0, power, torch.full_like(power, -127))
    y = torch.ldexp(x, -power).abs_()
    r = torch.where(y <= 0.25, 0.0, torch.where(y < 0.75, 0.5, torch.where(y <= 1.25, 1.0, torch.where(
        y < 1.75, 1.5, torch.where(y <= 2.5, 2.0, torch.where(y < 3.5, 3.0, torch.where(y <= 5.0, 4.0, 6.0)))))))
    r = torch.ldexp(torch.where(x < 0, -r, r), power)
    return r.reshape(shape)


def run(st):
    case, op = st["case"], st["case"]["op"]
    if not own:
        if op == "quantize":
            return dict(values=_rounded(st["W"].float()).to(torch.bfloat16))
        if op == "logits":
            return dict(logits=torch.matmul(_rounded(st["rows"].float()), st["W4"].T).to(DTYPES[case["out"]]))
        return {"sample": _plain_sample, "top": _plain_top, "distill": _plain_distill}[op](st)
    cai = st["cai"]
    if op == "sample":
        cai.cai_sample_rows(st["logits"], st["u"], st["token"], st["prob"], temperature=st["t"],
                            top_k=st["k"], top_p=st["p"], min_p=st["m"])
        return dict(token=st["token"], prob=st["prob"])
    if op == "top":
        cai.cai_top_rows(st["logits"], st["values"], st["index"], st["lse"], temperature=case["tau"])
        return dict(values=st["values"], index=st["index"], lse=st["lse"])
    if op == "distill":
        teacher = dict(top_lse=st["lse"], weight=st["weight"], temperature=case["tau"])
        if case["fused"]:
            cai.cai_distill_loss(st["logits"], st["values"], st["index"], st["loss"], st["stats"],
                                 grad=st["grad"], **teacher)
        else:
            cai.cai_distill_loss(st["logits"], st["values"], st["index"], st["loss"], st["stats"], **teacher)
            cai.cai_distill_backward(st["logits"], st["values"], st["index"], st["stats"], st["upstream"],
                                     st["grad"], **teacher)
        return dict(loss=st["loss"], stats=st["stats"], grad=st["grad"])
    if op == "quantize":
        cai.cai_mx4_update(st["head"].handle, st["W"], values=st["rounded"])
        return dict(values=st["rounded"])
    cai.cai_mx4_logits(st["head"].handle, st["rows"], st["out"])
    return dict(logits=st["out"])


# ------------------------------------------------------------------- bounds --

def work(case):
    op, V = case["op"], case["V"]
    if op == "quantize":
        n = float(V) * case["H"]
        # The weight in, its codes, scales and values out.
        return dict(bytes=n * (4 if case["dtype"] == "f32" else 2) + n * (0.5 + 1 / 32) + 2 * n, flops=2 * n)
    M = case["M"]
    if op == "logits":
        H = case["H"]
        out = (4.0 if case["out"] == "f32" else 2.0) * M * V
        return dict(bytes=V * H * (0.5 + 1 / 32) + 2.0 * M * H + out, flops=2.0 * V * H * M)
    size = 4.0 if case["dtype"] == "f32" else 2.0
    if op == "sample":
        # One exponential and a comparison for each logit.
        return dict(bytes=size * M * V + 28.0 * M, flops=4.0 * M * V)
    if op == "top":
        return dict(bytes=size * M * V + 8.0 * M * case["K"] + 4.0 * M, flops=4.0 * M * V)
    read = M - M // 8  # rows without weight need not be read
    return dict(bytes=size * (read + M) * V + 8.0 * M * case["K"] + 24.0 * M, flops=8.0 * read * V)


# ------------------------------------------------------------ 64-bit values --

def _exact_rounded(x):
    """By search among the E2M1 values' midpoints, in 64 bits."""
    b = x.double().reshape(-1, 32)
    high = b.abs().amax(1, keepdim=True)
    powers = torch.tensor([2.0 ** k for k in range(-125, 128)], dtype=torch.float64, device=x.device)
    # high is in [2^k, 2^(k+1)): the scale is 2^(k-2), 2^-127 at least.
    scale = torch.cat([powers[:1], powers])[torch.bucketize(high, powers, right=True)] / 4.0
    y = b / scale
    values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    middle = (values[1:] + values[:-1]) / 2
    low, upper = torch.bucketize(y.abs(), middle), torch.bucketize(y.abs(), middle, right=True)
    code = torch.where(low % 2 == 0, low, upper)  # differ at ties only; the even one
    r = torch.sign(y) * values[code] * scale
    return torch.where(high > 0, r, torch.zeros_like(r)).reshape(x.shape)


def exact(case, seed):
    op, st = case["op"], _inputs(case, seed)
    if op == "quantize":
        return dict(values=torch.cat([_exact_rounded(part) for part in st["W"].split(16384)]))
    if op == "logits":
        if 2.0 * case["M"] * case["V"] * case["H"] > 2e12:
            return None  # too long in 64 bits
        rows = _exact_rounded(st["rows"])
        return dict(logits=torch.cat([rows @ _exact_rounded(part).T for part in st["W"].split(16384)], 1))
    parts = []
    step = max(1, (1 << 26) // case["V"])
    for r in range(0, case["M"], step):
        part = {n: v[r:r + step] for n, v in st.items() if v is not None}
        parts.append({"sample": _exact_sample, "top": _exact_top, "distill": _exact_distill}[op](case, part))
    return {n: None if parts[0][n] is None else torch.cat([q[n] for q in parts]) for n in parts[0]}


def _exact_sample(case, st):
    z, t = st["logits"].double(), st["t"].double()
    greedy = t == 0
    plain = torch.softmax(z, 1)
    prob = torch.softmax(z / torch.where(greedy, torch.ones_like(t), t)[:, None], 1)
    sp, index = torch.sort(z, dim=1, descending=True, stable=True)
    sp = prob.gather(1, index)
    place = torch.arange(z.shape[1], device=z.device)[None]
    k = torch.where(st["k"] > 0, st["k"], torch.full_like(st["k"], z.shape[1]))[:, None]
    sp = sp * ((place < k) & (sp >= st["m"].double().clamp(max=1)[:, None] * sp[:, :1]))
    p = st["p"].double()[:, None]
    before = torch.cumsum(sp, 1) - sp
    sp = sp * ((p >= 1) | (before < p * sp.sum(1, keepdim=True)))
    kept = torch.zeros_like(prob).scatter_(1, index, sp)
    total = kept.sum(1, keepdim=True)
    token = torch.searchsorted(torch.cumsum(kept, 1), st["u"].double()[:, None] * total, right=True)
    at = torch.where(greedy[:, None], index[:, :1], token.clamp(max=z.shape[1] - 1))
    out = torch.where(greedy[:, None], plain.gather(1, at), kept.gather(1, at) / total)
    return dict(token=None, prob=out[:, 0])


def _exact_top(case, st):
    z = st["logits"].double()
    values = torch.topk(z, min(case["K"], case["V"]), 1).values
    return dict(values=values, index=None, lse=torch.logsumexp(z / case["tau"], 1))


def _exact_distill(case, st):
    tau = case["tau"]
    x = st["logits"].double() / tau
    M, V = x.shape
    teacher = torch.full((M, V + 1), -math.inf, dtype=torch.float64, device=x.device)
    index = st["index"].long()
    teacher.scatter_(1, torch.where(index < 0, torch.full_like(index, V), index), st["values"].double() / tau)
    teacher = teacher[:, :V]
    live = (st["weight"] != 0) & (index >= 0).any(1)
    chosen = torch.isfinite(teacher)
    norm = st["lse"].double() if case["tail"] else torch.logsumexp(teacher, 1)
    logq = teacher - norm[:, None]
    q = torch.exp(logq)
    lse = torch.logsumexp(x, 1)
    lse_rest = torch.logsumexp(torch.where(chosen, torch.full_like(x, -math.inf), x), 1)
    logp = x - lse[:, None]
    kl = torch.where(chosen, q * (logq - logp), torch.zeros_like(q)).sum(1)
    g = torch.exp(logp) - q  # the classes of the record
    w = st["weight"].double()
    if case["tail"]:
        rest = (1 - q.sum(1)).clamp(min=0)
        kl = kl + torch.where(rest > 0, rest * (torch.log(rest) - lse_rest + lse), torch.zeros_like(rest))
        inner = torch.exp(x - lse_rest[:, None])
        g = torch.where(chosen, g, torch.exp(logp) - rest[:, None] * inner)
    up = w if case["fused"] else w * st["upstream"].double()
    g = torch.where(live[:, None], g * (up * tau)[:, None], torch.zeros_like(g))
    none = torch.zeros_like(lse)
    return dict(loss=torch.where(live, w * tau * tau * kl, none),
                stats=torch.stack([torch.where(live, lse, none), torch.where(live, lse_rest, none)], 1), grad=g)
