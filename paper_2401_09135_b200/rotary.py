"""alsgd_rope as one differentiable function of torch tensors.

The call itself is binding.Rotary's; the backward pass is the same call the other way round.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as B


def _laid_out(t):
    """A gradient that arrives broadcast, transposed, or as a part of something larger that starts anywhere."""
    if t is None:
        return None
    unit = 16 // t.element_size()
    if t.stride(3) != 1 or any(s % unit for s in t.stride()[:3]) or t.data_ptr() % 16:
        return t.clone(memory_format=torch.contiguous_format)
    return t


def _like(t):
    return None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device)


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, q, k, positions):
        q_out, k_out = _like(q), _like(k)
        plan.alsgd_rope(q, k, q_out, k_out, positions=positions)
        ctx.plan = plan
        ctx.save_for_backward(positions)
        return q_out, k_out

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        positions, = ctx.saved_tensors
        # what needs no gradient is not turned back
        dq, dk = (_laid_out(t) if needed else None for t, needed in zip((dq, dk), ctx.needs_input_grad[1:3]))
        dq_in, dk_in = _like(dq), _like(dk)
        ctx.plan.alsgd_rope(dq, dk, dq_in, dk_in, positions=positions, inverse=True)
        return None, dq_in, dk_in, None


def rotate(plan: B.Rotary, q, k, positions=None):
    """q and k [batch, position, head, dim] at their positions, with gradients; second derivatives raise.  k is None, and so is its
    result, where the plan has no key heads or q is turned alone."""
    return _Rotate.apply(plan, q, k, positions)
