"""Losses over the vocabulary for many rows, gathered: which ones take part is counted in time that grows with the rows."""
import pytest
import torch

from paper_2401_09135_b200 import binding as B
from test_gpu_vocab import backward, forward, plan_of
from vocab_ref import Problem, off_by

pytestmark = pytest.mark.gpu


def overlapping(rows, dim):
    """Rows that share elements are gathered, however short the pass."""
    return torch.randn(8 * rows + dim, device="cuda").bfloat16().as_strided((rows, dim), (8, 1))


@pytest.mark.parametrize("top", [0, 3])
@pytest.mark.parametrize("rows", [513, 32704, 32768, 32769, 65599, 70001])
def test_rows_are_found_in_their_places(rows, top):
    p = Problem(rows, 50, 16, top=top, seed=rows, left_out=0.4)
    x = overlapping(rows, 16)
    p.x = x.contiguous()
    plan = plan_of(p)
    loss, lse = forward(plan, p, x=x)
    p.solve(lse=lse, gathered=True)
    assert off_by(loss, p.loss, p.loss_off) <= 1 and off_by(lse, p.lse, p.lse_off) <= 1
    dx, dw = backward(plan, p, lse, x=x)
    assert off_by(dx, p.dx, p.dx_off) <= 1 and off_by(dw, p.dw, p.dw_off) <= 1


def test_twice_the_rows_take_twice_the_time():
    """One word and narrow rows, so that gathering is what there is: twice the time, and four times if every block looked at all."""
    times = []
    for rows in (1 << 21, 1 << 22):
        x, w = torch.randn(1, 8, device="cuda").bfloat16().expand(rows, 8), torch.randn(1, 8, device="cuda").bfloat16()
        target = torch.arange(rows, device="cuda") % 3 - 1                 # a third of the rows takes part
        loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        plan = B.VocabLoss(rows, 1, 8)
        best = float("inf")
        for _ in range(4):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            start.record()
            for _ in range(3):
                plan.alsgd_xent_fwd(x, w, target, loss, lse)
            end.record()
            end.synchronize()
            best = min(best, start.elapsed_time(end))
        times.append(best)
    assert times[1] < 2.8 * times[0]
