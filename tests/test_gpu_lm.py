"""The small language model end to end: attention with its bias, clipping, inner and server steps together."""
import math

import pytest
import torch

from attn_ref import Case
from paper_2401_09135_b200 import binding as B
from paper_2401_09135_b200 import lm
from paper_2401_09135_b200.attention import attend

pytestmark = pytest.mark.gpu


def test_training_learns_the_lag():
    before, after, updates, share, theta = lm.run(total_local_steps=800)
    assert before > 0.9 * math.log(lm.VOCAB)
    # the noise alone (5 %) costs about 0.05 (log 20 + log 64) + 0.95 log(1 / 0.95) = 0.4; a model without attention stays at chance
    assert after < 0.5 * math.log(lm.VOCAB)
    assert updates > 0 and bool(torch.isfinite(theta).all())


def test_the_same_seed_gives_the_same_model():
    """No atomics, fixed summation orders: two runs end with the same bits."""
    a, b = (lm.run(total_local_steps=120) for _ in range(2))
    assert a[1] == b[1] and torch.equal(a[4], b[4])


@pytest.mark.parametrize("buckets", [0, 32])
def test_autograd_function(buckets):
    """attend() against the same graph in 64-bit PyTorch.  The tolerance is the backward test's, on norms: two roundings of
    2^-8 for each product chain, averaged over many elements, stay below 2^-7."""
    c = Case(batch=2, len_q=140, heads_q=4, heads_kv=2, buckets=buckets, kv_len=(140, 77))
    q, k, v, w, table, lens = c.inputs()
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)] + ([table.clone().requires_grad_(True)] if buckets else [])
    plan = B.Attention(2, 140, 140, 4, 2, 64, buckets=buckets)
    out = attend(plan, *leaves[:3], table=leaves[3] if buckets else None, kv_len=lens)
    (out * w).sum().backward()
    wide = [t.detach().double().requires_grad_(True) for t in leaves]
    total = 0.0
    for b in range(2):
        for h in range(4):
            x = c.scale * wide[0][b, :, h] @ wide[1][b, :, h // 2].T
            _, _, _, _, ok, at = c.head(q, k, v, table, b, h)
            if buckets:
                x = x + wide[3][h][at]
            p = torch.softmax(x.masked_fill(~ok, -math.inf), 1)
            total = total + ((p @ wide[2][b, :, h // 2]) * w[b, :, h].double()).sum()
    total.backward()
    for a, b in zip(leaves, wide):
        assert float((a.grad.double() - b.grad).norm()) <= 2.0 ** -7 * float(b.grad.norm())


def test_a_broadcast_gradient_is_laid_out():
    c = Case(batch=2, len_q=40)
    q, k, v, _, _, _ = c.inputs()
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
    attend(B.Attention(2, 40, 40, 2, 2, 64), *leaves).sum().backward()
    # the sum of o over a row's elements has dv_j = sum_i p_ij for every element: the columns of v's gradient agree
    assert bool((leaves[2].grad == leaves[2].grad[..., :1]).all())
