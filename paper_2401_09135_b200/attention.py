"""alsgd_attn_fwd / alsgd_attn_bwd as one differentiable function of torch tensors.

The calls themselves are binding.Attention's; this module only keeps what the backward pass needs and hands out the
results' memory.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as B


class _Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, plan, q, k, v, table, kv_len):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[0], q.shape[2], q.shape[1], dtype=torch.float32, device=q.device)
        plan.alsgd_attn_fwd(q, k, v, out, lse, table=table, kv_len=kv_len)
        ctx.plan = plan
        ctx.save_for_backward(q, k, v, table, kv_len, out, lse)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, table, kv_len, out, lse = ctx.saved_tensors
        # a gradient that arrives broadcast over positions or within a head (a sum's, say), transposed, or as a part of
        # something larger that starts anywhere is laid out first
        if dout.stride(3) != 1 or dout.stride(1) == 0 or any(s % 8 for s in dout.stride()[:3]) or dout.data_ptr() % 16:
            dout = dout.clone(memory_format=torch.contiguous_format)
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        dtable = None if table is None else torch.empty_like(table)
        ctx.plan.alsgd_attn_bwd(q, k, v, out, lse, dout, dq, dk, dv, table=table, dtable=dtable, kv_len=kv_len)
        return None, dq, dk, dv, dtable, None


def attend(plan: B.Attention, q, k, v, table=None, kv_len=None):
    """Attention of bf16 operands [batch, position, head, dim] with gradients for q, k, v and the bias table; second derivatives
    raise.  `plan` belongs to one stream: its workspace is used by every backward pass through it."""
    return _Attend.apply(plan, q, k, v, table, kv_len)
