"""attention.attend as a part of autograd: what arrives as the result's gradient, and derivatives of derivatives.

On the CPU with a plan that does the sums in 64-bit PyTorch and takes and refuses operands as the library does; on the GPU
with the library's."""
import math

import pytest
import torch

from paper_2401_09135_b200 import binding as B
from paper_2401_09135_b200.attention import attend

SHAPE = (2, 40, 2, 64)


def attention(q, k, v):
    x = torch.einsum("bihd,bjhd->bhij", q, k) * q.shape[-1] ** -0.5
    ahead = torch.ones(q.shape[1], k.shape[1], dtype=torch.bool, device=q.device).triu(1)
    return torch.einsum("bhij,bjhd->bihd", torch.softmax(x.masked_fill(ahead, -math.inf), -1), v)


class HostPlan:
    """Causal attention of SHAPE on host tensors."""

    def operand(self, t, output=False):
        assert t.dtype is torch.bfloat16 and t.shape == SHAPE and t.stride(3) == 1
        bad = t.data_ptr() % 16
        for i in range(3):
            if t.shape[i] > 1:
                bad = bad or t.stride(i) % 8 or (t.stride(i) == 0 and (output or i == 1))
        if bad:
            raise B.AlsgdError(B.E_ARG, "operand")

    def alsgd_attn_fwd(self, q, k, v, out, lse, table=None, kv_len=None):
        for t in (q, k, v):
            self.operand(t)
        self.operand(out, True)
        out.copy_(attention(q.double(), k.double(), v.double()))

    def alsgd_attn_bwd(self, q, k, v, out, lse, dout, dq, dk, dv, table=None, dtable=None, kv_len=None):
        for t in (q, k, v, out, dout):
            self.operand(t)
        with torch.enable_grad():
            wide = [t.detach().double().requires_grad_(True) for t in (q, k, v)]
            grads = torch.autograd.grad(attention(*wide), wide, dout.double())
        for t, g in zip((dq, dk, dv), grads):
            self.operand(t, True)
            t.copy_(g)


PLACES = [pytest.param("cpu", id="host"), pytest.param("cuda", id="device", marks=pytest.mark.gpu)]


def plan_on(device):
    return HostPlan() if device == "cpu" else B.Attention(*SHAPE[:2], SHAPE[1], SHAPE[2], SHAPE[2], SHAPE[3])


def leaves_on(device, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(SHAPE, generator=g).bfloat16().to(device).requires_grad_(True) for _ in range(3)]


def gradients(device, loss):
    leaves = leaves_on(device)
    return torch.autograd.grad(loss(attend(plan_on(device), *leaves)), leaves)


@pytest.mark.parametrize("device", PLACES)
@pytest.mark.parametrize("dims", [(0,), (1,), (2,), (3,), (0, 1), (1, 2), (0, 2), (2, 3), (0, 1, 2), (0, 1, 2, 3)])
def test_sums_over_some_dimensions(device, dims):
    """The gradient of a sum arrives with steps of zero over what was summed; the same numbers laid out give the same bits."""
    w = torch.randn(SHAPE, generator=torch.Generator().manual_seed(1)).to(device)
    w = w.mean(dims, keepdim=True).bfloat16()
    got = gradients(device, lambda o: (o.sum(dims, keepdim=True) * w).sum())

    class LaidOut(torch.autograd.Function):
        @staticmethod
        def forward(ctx, o):
            return o.sum(dims, keepdim=True)

        @staticmethod
        def backward(ctx, g):
            return g.expand(SHAPE).clone(memory_format=torch.contiguous_format)
    want = gradients(device, lambda o: (LaidOut.apply(o) * w).sum())
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("device", PLACES)
@pytest.mark.parametrize("shift", [1, 3, 4])
def test_a_gradient_that_is_not_aligned(device, shift):
    """Behind other elements of one vector the gradient is contiguous and starts anywhere."""
    n = math.prod(SHAPE)
    w = torch.randn(n + shift, generator=torch.Generator().manual_seed(2)).bfloat16().to(device)
    got = gradients(device, lambda o: (torch.cat([o.new_zeros(shift), o.flatten()]) * w).sum())
    want = gradients(device, lambda o: (o.flatten() * w[shift:].clone()).sum())
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("device", PLACES)
def test_gradients_turned_round(device):
    """Heads ahead of positions, and elements of a head that are not side by side."""
    w = torch.randn(SHAPE, generator=torch.Generator().manual_seed(3)).bfloat16().to(device)
    want = gradients(device, lambda o: (o * w).sum())
    for order in ((0, 2, 1, 3), (3, 1, 2, 0), (0, 1, 3, 2)):
        turned = w.permute(order).contiguous()
        got = gradients(device, lambda o: (o.permute(order) * turned).sum())
        assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("device", PLACES)
def test_second_derivatives_are_refused(device):
    """The backward pass is not differentiable: a gradient penalty has to raise, not lose its part of the gradient."""
    leaves = leaves_on(device)
    loss = (attend(plan_on(device), *leaves).float() ** 2).sum()
    first = torch.autograd.grad(loss, leaves, create_graph=True)
    with pytest.raises(RuntimeError):
        (loss + sum((g.float() ** 2).sum() for g in first)).backward()
