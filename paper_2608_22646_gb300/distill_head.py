"""A 4-bit LM head trained on a teacher's records, then sampled from.

    python -m paper_2608_22646_gb300.distill_head --workload toy --steps 60

The operators around the decoding head, together as a program uses them, on a
seeded synthetic weight and hidden states (``synth``):

1. the teacher's bf16 head makes logits, ``cai_top_rows`` keeps its K largest
   and its log-sum-exp of every row;
2. a copy of the weight, held in 32 bits, is re-quantised every step
   (``cai_mx4_update``), makes the student's logits (``cai_mx4_logits``) and is
   moved by the gradient of the distillation loss (``cai_distill_loss``,
   ``cai_distill_backward`` through autograd, straight through the rounding);
3. a block is decoded from the trained head: the masked positions' tokens are
   drawn at a temperature within a nucleus (``cai_sample_rows``) and the
   confident ones kept, step by step, until none is masked.

Prints the loss and how often the student's likeliest token is the teacher's,
before and after, and the decoded block's steps.
"""
from __future__ import annotations

import argparse
import json
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch
from torch.autograd.function import once_differentiable

import paper_2608_22646_gb300 as cai


class DistillLoss(torch.autograd.Function):
    """Each row's distillation loss of ``logits`` [M, V] against a teacher's
    record, for autograd: the forward call computes losses and statistics, the
    backward call the gradient times whatever reaches each row's loss."""

    @staticmethod
    def forward(ctx, logits, record, temperature, weight):
        if ctx.needs_input_grad[3]:
            raise ValueError("weight: the loss has a gradient by the logits only")
        M = logits.shape[0]
        loss = torch.empty(M, dtype=torch.float32, device=logits.device)
        stats = torch.empty((M, 2), dtype=torch.float32, device=logits.device)
        values, index, lse = record
        cai.cai_distill_loss(logits, values, index, loss, stats, top_lse=lse, temperature=temperature,
                             weight=weight)
        ctx.save_for_backward(logits, values, index, stats, lse, weight)
        ctx.temperature = temperature
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_loss):
        logits, values, index, stats, lse, weight = ctx.saved_tensors
        grad = torch.empty_like(logits)
        cai.cai_distill_backward(logits, values, index, stats, grad_loss.float().contiguous(), grad,
                                 top_lse=lse, temperature=ctx.temperature, weight=weight)
        return grad, None, None, None


class Mx4Linear(torch.autograd.Function):
    """Logits of ``rows`` from the 4-bit head of ``W``.  Gradients pass straight
    through the rounding: by W it is the gradient times the rows as given, by
    the rows the gradient times the values that W's codes stand for."""

    @staticmethod
    def forward(ctx, W, rows, head):
        values = torch.empty(W.shape, dtype=torch.bfloat16, device=W.device) if ctx.needs_input_grad[1] else None
        cai.cai_mx4_update(head, W.detach(), values)
        out = torch.empty((rows.shape[0], W.shape[0]), dtype=torch.float32, device=rows.device)
        cai.cai_mx4_logits(head, rows, out)
        ctx.save_for_backward(rows, values)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, grad):
        rows, values = ctx.saved_tensors
        by_W = grad.T @ rows.float() if ctx.needs_input_grad[0] else None
        by_rows = (grad @ values.float()).to(rows.dtype) if ctx.needs_input_grad[1] else None
        return by_W, by_rows, None


def record_of(logits, K, temperature):
    """The teacher's record of every row: K largest logits, their tokens, and
    the row's log-sum-exp at the temperature."""
    M = logits.shape[0]
    values = torch.empty((M, K), dtype=torch.float32, device=logits.device)
    index = torch.empty((M, K), dtype=torch.int32, device=logits.device)
    lse = torch.empty(M, dtype=torch.float32, device=logits.device)
    cai.cai_top_rows(logits, values, index, lse, temperature=temperature)
    return values, index, lse


def decode_block(head, hidden, threshold=0.3, temperature=0.7, top_p=0.95, seed=0):
    """Tokens of a block of masked positions: ``hidden(t)`` [P, H] bf16 are the
    rows at step t.  Every step draws a token for every masked position and
    keeps those whose probability reaches the threshold, the likeliest at
    least; rows without a softmax (probability NaN, their token as
    cai_sample_rows defines it) are kept once no other is left.  So there are at
    most P steps.  Returns (tokens [P] int32, steps)."""
    first = hidden(0)
    P, device = first.shape[0], first.device
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    tokens = torch.full((P,), cai.CAI_MASK_TOKEN, dtype=torch.int32, device=device)
    steps = 0
    while bool((tokens == cai.CAI_MASK_TOKEN).any()):
        at = torch.nonzero(tokens == cai.CAI_MASK_TOKEN).flatten()
        rows = hidden(steps)[at].contiguous()
        n = rows.shape[0]
        logits = torch.empty((n, head.V), dtype=torch.bfloat16, device=device)
        cai.cai_mx4_logits(head, rows, logits)
        drawn = torch.empty(n, dtype=torch.int32, device=device)
        prob = torch.empty(n, dtype=torch.float32, device=device)
        settings = dict(temperature=torch.full((n,), temperature, device=device),
                        top_p=torch.full((n,), top_p, device=device))
        cai.cai_sample_rows(logits, torch.rand(n, generator=g, device=device), drawn, prob, **settings)
        score = torch.nan_to_num(prob, nan=-1.0)
        keep = score >= score.max().clamp(max=threshold)
        tokens[at[keep]] = drawn[keep]
        steps += 1
    return tokens, steps


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workload", default="toy")
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--top", type=int, default=64, help="the teacher's logits kept of a row")
    ap.add_argument("--temperature", type=float, default=2.0)
    ap.add_argument("--lr", type=float, default=2e-4)
    args = ap.parse_args(argv)
    import synth

    wl = synth.WORKLOADS[args.workload]
    W = synth.lm_head_weight(wl.V, wl.H, seed=wl.seed_w, device="cuda")
    hs = synth.HiddenStates(wl, W, "calibrated")

    def rows(step):  # [B P, H] of some block and step of a generation
        return hs(step % wl.n_blocks, step % wl.T).reshape(-1, wl.H).contiguous()

    student = torch.nn.Parameter(W.float())
    optimiser = torch.optim.Adam([student], lr=args.lr)
    held = rows(0)
    with cai.cai_mx4_init(student.detach(), held.shape[0]) as head:

        def evaluate():
            teacher = (held @ W.T).float()
            logits = Mx4Linear.apply(student.detach(), held, head)
            loss = DistillLoss.apply(logits, record_of(teacher, args.top, args.temperature), args.temperature, None)
            return float(loss.mean()), float((logits.argmax(1) == teacher.argmax(1)).float().mean())

        before = evaluate()
        for step in range(args.steps):
            x = rows(step)
            record = record_of(x @ W.T, args.top, args.temperature)
            logits = Mx4Linear.apply(student, x, head)
            loss = DistillLoss.apply(logits, record, args.temperature, None).mean()
            optimiser.zero_grad()
            loss.backward()
            optimiser.step()
        after = evaluate()
        tokens, steps = decode_block(head, lambda t: hs(0, min(t, wl.T - 1))[0])
        print(json.dumps({"workload": wl.name, "loss": [before[0], after[0]],
                          "same_likeliest_token": [before[1], after[1]], "block_steps": steps,
                          "tokens": tokens[:8].tolist()}))
    return 0


if __name__ == "__main__":
    sys.exit(main())
