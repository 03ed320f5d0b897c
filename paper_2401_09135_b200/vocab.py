"""alsgd_xent_* and alsgd_distill_* as differentiable functions of torch tensors: losses over a vocabulary, row by row, without
its logits.

The calls themselves are binding.VocabLoss's; this module only keeps what the backward pass needs and hands out the results'
memory.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as B


class _Loss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, x, w, index, teacher):
        loss, lse = (torch.empty(x.shape[0], dtype=torch.float32, device=x.device) for _ in range(2))
        if teacher is None:
            plan.alsgd_xent_fwd(x, w, index, loss, lse)
        else:
            plan.alsgd_distill_fwd(x, w, index, teacher, loss, lse)
        ctx.plan = plan
        ctx.save_for_backward(x, w, index, teacher, lse)
        return loss

    @staticmethod
    @once_differentiable
    def backward(ctx, dloss):
        x, w, index, teacher, lse = ctx.saved_tensors
        # a frozen embedding, or rows that nothing is learnt through, has no gradient made for it
        dx, dw = (torch.empty(t.shape, dtype=t.dtype, device=t.device) if needed else None for t, needed in zip((x, w), ctx.needs_input_grad[1:3]))
        if dx is None and dw is None:
            return None, None, None, None, None
        if teacher is None:
            ctx.plan.alsgd_xent_bwd(x, w, index, lse, dloss, dx, dw)
        else:
            ctx.plan.alsgd_distill_bwd(x, w, index, teacher, lse, dloss, dx, dw)
        return None, dx, dw, None, None


def cross_entropy(plan: B.VocabLoss, x, w, target):
    """Cross entropy of every row of x [rows, dim] against its target over the words w [vocab, dim]; 0 where the target is no
    word.  Gradients for x and w; second derivatives raise."""
    return _Loss.apply(plan, x, w, target, None)


def distill(plan: B.VocabLoss, x, w, index, teacher):
    """Divergence of a teacher's highest logits (words `index`, logits `teacher`, both [rows, top]) from every row's softmax.
    Gradients for x and w; second derivatives raise."""
    return _Loss.apply(plan, x, w, index, teacher)
