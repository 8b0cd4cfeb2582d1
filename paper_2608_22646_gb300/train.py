"""Training around the decoding head: autograd functions and an optimiser over
the library's operators.

* ``TokenLogp``, ``PolicyLoss``, ``PreferenceLoss``: log-probabilities of given
  tokens, the clipped policy loss on drawn ones, the preference loss of pairs
  of sequences;
* ``NormRows``: the layer norm or RMS norm in front of a head;
* ``AdamW``: a step over all parameters at once, states in 32 or 8 bits.

The functions are once differentiable, and only by what their documentation
names: another input that wants a gradient is an error.  They can be captured into
a CUDA graph; torch asks that no uncaptured graph of the same leaves is alive then.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

import paper_2608_22646_gb300 as cai


def _only(ctx, *differentiable: int) -> None:
    for i, wanted in enumerate(ctx.needs_input_grad):
        if wanted and i not in differentiable:
            raise ValueError(f"{type(ctx).__name__[:-8]}: input {i} has no gradient here")


def _floats(n, like) -> torch.Tensor:
    return torch.empty(n, dtype=torch.float32, device=like.device)


def _rows(x) -> torch.Tensor:
    """``x`` [..., H] as rows whose elements are adjacent and which do not overlap."""
    rows = x.reshape(-1, x.shape[-1])
    return rows if rows.stride(1) == 1 and (rows.shape[0] <= 1 or rows.stride(0) >= rows.shape[1]) else rows.contiguous()


class TokenLogp(torch.autograd.Function):
    """``TokenLogp.apply(logits, token, temperature)``: each row's
    log-probability [M] of its ``token`` (int32 [M]; outside [0, V): 0),
    differentiable by the logits [M, V]."""

    @staticmethod
    def forward(ctx, logits, token, temperature=1.0):
        _only(ctx, 0)
        M = logits.shape[0]
        logp, stats = _floats(M, logits), _floats((M, 2), logits)
        cai.cai_token_logp(logits, token, logp, stats, temperature=temperature)
        ctx.save_for_backward(logits, token, stats)
        ctx.temperature = temperature
        return logp

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_logp):
        logits, token, stats = ctx.saved_tensors
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        cai.cai_token_logp_backward(logits, token, stats, grad_logp.float().contiguous(), grad,
                                    temperature=ctx.temperature)
        return grad, None, None


class PolicyLoss(torch.autograd.Function):
    """``loss, logp = PolicyLoss.apply(logits, token, advantage, old_logp,
    ref_logp, weight, settings)``: each row's clipped policy loss, differentiable
    by the logits, and its log-probability, which is not.  ``settings``: a dict
    of cai_policy_loss's temperature, clip_low, clip_high and kl."""

    @staticmethod
    def forward(ctx, logits, token, advantage, old_logp=None, ref_logp=None, weight=None, settings=None):
        _only(ctx, 0)
        settings = dict(settings or {})
        M = logits.shape[0]
        loss, logp, slope, stats = (_floats(n, logits) for n in (M, M, M, (M, 2)))
        cai.cai_policy_loss(logits, token, advantage, loss, logp, stats, slope, old_logp=old_logp, ref_logp=ref_logp,
                            weight=weight, **settings)
        ctx.save_for_backward(logits, token, stats, slope)
        ctx.temperature = settings.get("temperature", 1.0)
        ctx.mark_non_differentiable(logp)
        return loss, logp

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_loss, _):
        logits, token, stats, slope = ctx.saved_tensors
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        cai.cai_policy_backward(logits, token, stats, slope, grad_loss.float().contiguous(), grad,
                                temperature=ctx.temperature)
        return (grad,) + (None,) * 6


class PreferenceLoss(torch.autograd.Function):
    """``loss, margin = PreferenceLoss.apply(logp, offsets, ref_logp, weight,
    beta, smoothing)``: the preference loss [pairs] of pairs of sequences from
    their tokens' log-probabilities ``logp`` [M], differentiable by these, and
    the margins, which are not.  ``offsets``: see cai_preference_loss."""

    @staticmethod
    def forward(ctx, logp, offsets, ref_logp=None, weight=None, beta=0.1, smoothing=0.0):
        _only(ctx, 0)
        pairs = offsets.shape[0] // 2
        loss, margin = _floats(pairs, logp), _floats(pairs, logp)
        cai.cai_preference_loss(logp, offsets, loss, margin, ref_logp=ref_logp, weight=weight, beta=beta,
                                smoothing=smoothing)
        ctx.save_for_backward(logp, offsets, ref_logp, weight)
        ctx.settings = dict(beta=beta, smoothing=smoothing)
        ctx.mark_non_differentiable(margin)
        return loss, margin

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_loss, _):
        logp, offsets, ref_logp, weight = ctx.saved_tensors
        pairs = offsets.shape[0] // 2
        grad = torch.empty_like(logp)
        cai.cai_preference_loss(logp, offsets, _floats(pairs, logp), _floats(pairs, logp), grad, ref_logp=ref_logp,
                                weight=weight, grad_loss=grad_loss.float().contiguous(), **ctx.settings)
        return (grad,) + (None,) * 5


class NormRows(torch.autograd.Function):
    """``NormRows.apply(x, weight, bias, kind, eps)``: the norm of the rows of
    ``x`` [..., H], differentiable by x, weight and bias (the last two [H] or
    None); ``kind``: CAI_NORM_LAYER or CAI_NORM_RMS."""

    @staticmethod
    def forward(ctx, x, weight=None, bias=None, kind=cai.CAI_NORM_LAYER, eps=1e-5):
        _only(ctx, 0, 1, 2)
        rows = _rows(x)
        y = torch.empty(rows.shape, dtype=x.dtype, device=x.device)
        stats = _floats((rows.shape[0], 2), x)
        cai.cai_norm_rows(rows, y, stats, weight=weight, bias=bias, kind=kind, eps=eps)
        ctx.save_for_backward(x, weight, stats)
        ctx.kind, ctx.bias = kind, None if bias is None else bias.dtype
        return y.view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_y):
        x, weight, stats = ctx.saved_tensors
        by_x, by_weight, by_bias = ctx.needs_input_grad[:3]
        rows, grad_y = _rows(x), _rows(grad_y)
        M, H = rows.shape
        out = [torch.empty((M, H), dtype=x.dtype, device=x.device) if by_x else None,
               torch.empty_like(weight) if by_weight else None,
               torch.empty(H, dtype=ctx.bias, device=x.device) if by_bias else None]
        space = None
        if by_weight or by_bias:
            space = torch.empty(cai.cai_norm_workspace(M, H), dtype=torch.uint8, device=x.device)
        cai.cai_norm_backward(rows, grad_y, stats, space, grad_x=out[0], grad_weight=out[1], grad_bias=out[2],
                              weight=weight, kind=ctx.kind)
        return (out[0].view(x.shape) if by_x else None, out[1], out[2], None, None)


class AdamW:
    """AdamW over ``params`` (contiguous CUDA parameters, float32 or bf16) with
    one launch a step for every kind of them.  ``state_bits`` 8 keeps the states
    as E4M3 in blocks of 32, a quarter of their bytes, rounded by a hash of
    ``seed``, the parameter's type and place, the step and the element.  ``copies``: {parameter: bf16 tensor} of
    float32 parameters whose rounded values are written along.  ``decay`` may be
    a function of a parameter.  Its handles live until ``close()`` or the end of a
    ``with``: freeing them synchronises the device, which an object that is dropped
    may not do at any time."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, decay=0.01, state_bits=32, copies=None, seed=0):
        self.params = list({id(p): p for p in params}.values())  # shared ones once
        self.lr, self.betas, self.eps, self.seed, self.state_bits = lr, tuple(betas), eps, seed, state_bits
        self.steps = 0
        copies = {id(k): v for k, v in (copies or {}).items()}
        self.state, kinds = [], {}
        for p in self.params:
            n, kw = p.numel(), dict(device=p.device)
            if state_bits == 32:
                s = dict(m=torch.zeros(n, **kw), v=torch.zeros(n, **kw))
            else:
                sizes = dict(m=n, v=n, m_scale=(n + 31) // 32, v_scale=(n + 31) // 32)
                s = {k: torch.zeros(c, dtype=torch.uint8, **kw) for k, c in sizes.items()}
            self.state.append(s)
            kinds.setdefault(p.dtype, []).append(
                (p, dict(param=p.detach(), copy=copies.get(id(p)), decay=decay(p) if callable(decay) else decay, **s)))
        self.groups = []  # of one dtype: gradients are all alike in a call
        for members in kinds.values():
            group = [p for p, _ in members]
            try:
                opt = cai.cai_adamw_init([t for _, t in members], state_bits)
            except Exception:
                self.close()  # the groups before
                raise
            self.groups.append((group, [p.data_ptr() for p in group], opt))

    def zero_grad(self) -> None:
        for p in self.params:
            p.grad = None

    @torch.no_grad()
    def step(self, grad_scale=None, lr_step=None) -> None:
        """A step of every parameter with a gradient.  ``grad_scale`` and
        ``lr_step``: see cai_adamw_step.  ``steps`` counts the calls that succeeded: a
        step that is refused is none, and moves no parameter.  (A captured one is counted
        once: who replays it with ``lr_step`` sets ``steps`` to its t before a
        state_dict().)"""
        # What one group alone could be refused for, before any group moves; settings
        # are the same for all, and looked at by the first one's call.
        step, work = self.steps + 1, []
        for params, places, opt in self.groups:
            for p, at, t in zip(params, places, opt.tensors):
                if p.data_ptr() != at or p.numel() != t["param"].numel():
                    raise RuntimeError("AdamW: a parameter has another storage than when the optimiser was made")
            work.append([None if p.grad is None else p.grad.to(p.dtype).contiguous() for p in params])
        for i, ((params, _, opt), grads) in enumerate(zip(self.groups, work)):
            # A group counts its tensors from 0: another seed, or the first of each would be
            # rounded alike.  (From the group's number alone, so that a loaded state goes on.)
            seed = (self.seed + 0x9e3779b9 * i) & 0xffffffff
            cai.cai_adamw_step(opt, grads, lr=self.lr, step=step, beta1=self.betas[0], beta2=self.betas[1],
                               eps=self.eps, seed=seed, grad_scale=grad_scale, lr_step=lr_step)
            # What autograd has kept of them is not what they are any more.
            for p, g, t in zip(params, grads, opt.tensors):
                if g is not None:
                    torch.autograd.graph.increment_version(p)
                    if t["copy"] is not None:
                        torch.autograd.graph.increment_version(t["copy"])
        self.steps = step

    def state_dict(self) -> dict:
        return dict(steps=self.steps, seed=self.seed, state_bits=self.state_bits,
                    state=[{k: v.clone() for k, v in s.items()} for s in self.state])

    def load_state_dict(self, saved: dict) -> None:
        if saved["state_bits"] != self.state_bits or len(saved["state"]) != len(self.state):
            raise ValueError("AdamW: a state of other parameters or of other bits")
        for s, t in zip(self.state, saved["state"]):
            for k in s:
                if t[k].shape != s[k].shape or t[k].dtype != s[k].dtype:
                    raise ValueError("AdamW: a state of other parameters")
        for s, t in zip(self.state, saved["state"]):
            for k in s:
                s[k].copy_(t[k])
        self.steps, self.seed = saved["steps"], saved["seed"]

    def close(self) -> None:
        for _, _, opt in self.groups:
            cai.cai_adamw_free(opt)

    def __enter__(self) -> "AdamW":
        return self

    def __exit__(self, *exc) -> None:
        self.close()
