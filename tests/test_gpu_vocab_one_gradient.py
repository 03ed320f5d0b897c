"""Backward passes of which only one gradient is wanted."""
import pytest
import torch

from paper_2401_09135_b200.vocab import cross_entropy, distill
from test_gpu_vocab import forward, plan_of
from vocab_ref import Problem

pytestmark = pytest.mark.gpu


def backward(plan, p, lse, dx, dw):
    if p.top:
        plan.alsgd_distill_bwd(p.x, p.w, p.index, p.teacher, lse, p.dloss, dx, dw)
    else:
        plan.alsgd_xent_bwd(p.x, p.w, p.index, lse, p.dloss, dx, dw)


# few rows in two parts, with dx's parts; both kinds of short passes; gathered; two pieces; several tiles of dim; dw in parts
SIZES = [(1, 1, 8), (20, 40000, 64), (90, 300, 136), (300, 5003, 384), (700, 1500, 896), (6000, 5000, 328), (16384, 8960, 64), (10604, 1240, 104), (3000, 9000, 520)]


@pytest.mark.parametrize("top", [0, 4])
@pytest.mark.parametrize("rows,vocab,dim", SIZES)
def test_one_gradient_has_the_bits_of_both(rows, vocab, dim, top):
    p = Problem(rows, vocab, dim, top=top, seed=rows, left_out=0.2)
    plan = plan_of(p)
    _, lse = forward(plan, p)
    want, got = [(torch.full_like(p.x, 7.0), torch.full_like(p.w, 7.0)) for _ in range(2)]
    backward(plan, p, lse, *want)
    backward(plan, p, lse, got[0], None)
    backward(plan, p, lse, None, got[1])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("rows,left_out", [(0, 0.0), (30, 2.0), (600, 2.0), (6000, 2.0)])
def test_one_gradient_without_rows(rows, left_out):
    p = Problem(rows, 12000 if rows > 600 else 700, 136, left_out=left_out)
    plan = plan_of(p)
    _, lse = forward(plan, p)
    dx, dw = torch.full_like(p.x, 7.0), torch.full_like(p.w, 7.0)
    backward(plan, p, lse, dx, None)
    backward(plan, p, lse, None, dw)
    assert not bool(dx.any()) and not bool(dw.any())


@pytest.mark.parametrize("top", [0, 3])
def test_autograd_makes_what_is_asked_for(top):
    """With frozen words no tensor of their size is made; with rows that need no gradient none of theirs."""
    p = Problem(400, 30000, 64, top=top, seed=1)
    plan = plan_of(p)
    losses = lambda x, w: distill(plan, x, w, p.index, p.teacher) if top else cross_entropy(plan, x, w, p.index)  # noqa: E731
    x, w = p.x.clone().requires_grad_(True), p.w.clone().requires_grad_(True)
    want = torch.autograd.grad(losses(x, w).mean(), (x, w))
    mean = losses(x, p.w).mean()
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    got, = torch.autograd.grad(mean, x)
    assert torch.equal(got, want[0]) and torch.cuda.max_memory_allocated() - before < p.w.numel()
    got, = torch.autograd.grad(losses(p.x, w).mean(), w)
    assert torch.equal(got, want[1])
    if top:
        # a teacher's logits are taken as they are
        logits = p.teacher.clone().requires_grad_(True)
        distill(plan, p.x, p.w, p.index, logits).mean().backward()
        assert logits.grad is None
