"""Losses over the vocabulary against the same in 64 bits: sizes around the tiles' edges, rows and entries that take no part,
steps, types, streams and graphs."""
import math

import pytest
import torch

from paper_2401_09135_b200 import binding as B
from paper_2401_09135_b200.vocab import cross_entropy, distill
from vocab_ref import Problem, off_by

pytestmark = pytest.mark.gpu


def plan_of(p):
    return B.VocabLoss(p.rows, p.vocab, p.dim, top=p.top, scale=p.scale, index_dtype=p.index.dtype,
                       teacher_dtype=None if p.teacher is None else p.teacher.dtype)


def forward(plan, p, x=None, w=None, stream=None):
    loss, lse = (torch.full((p.rows,), 7.0, device="cuda") for _ in range(2))
    x, w = p.x if x is None else x, p.w if w is None else w
    if p.top:
        plan.alsgd_distill_fwd(x, w, p.index, p.teacher, loss, lse, stream=stream)
    else:
        plan.alsgd_xent_fwd(x, w, p.index, loss, lse, stream=stream)
    return loss, lse


def backward(plan, p, lse, dloss=None, x=None, w=None, dx=None, dw=None, stream=None):
    x, w = p.x if x is None else x, p.w if w is None else w
    dx, dw = torch.full_like(p.x, 7.0) if dx is None else dx, torch.full_like(p.w, 7.0) if dw is None else dw
    dloss = p.dloss if dloss is None else dloss
    if p.top:
        plan.alsgd_distill_bwd(x, w, p.index, p.teacher, lse, dloss, dx, dw, stream=stream)
    else:
        plan.alsgd_xent_bwd(x, w, p.index, lse, dloss, dx, dw, stream=stream)
    return dx, dw


def check(p, dloss=None):
    plan = plan_of(p)
    loss, lse = forward(plan, p)
    p.solve(lse=lse, dloss=dloss)
    assert off_by(loss, p.loss, p.loss_off) <= 1 and off_by(lse, p.lse, p.lse_off) <= 1
    dx, dw = backward(plan, p, lse, dloss=dloss)
    assert off_by(dx, p.dx, p.dx_off) <= 1 and off_by(dw, p.dw, p.dw_off) <= 1
    assert B.alsgd_vocab_status() == 0
    return loss, lse, dx, dw


@pytest.mark.parametrize("rows,vocab,dim", [
    (1, 1, 8), (1, 300, 64), (2, 7, 16), (5, 256, 64), (64, 255, 72), (77, 257, 136), (128, 1000, 64), (129, 513, 200), (255, 2000, 256),
    (256, 640, 264), (257, 1024, 96), (300, 5003, 384), (513, 300, 520), (700, 1500, 896), (1000, 1280, 1032), (33, 32000, 384), (512, 700, 64), (5000, 300, 64), (2600, 64, 64), (3000, 1000, 520), (6000, 1, 8), (130, 300, 2056),
])
def test_labels(rows, vocab, dim):
    check(Problem(rows, vocab, dim, seed=rows))


@pytest.mark.parametrize("rows,vocab,dim,top", [
    (1, 1, 8, 1), (1, 300, 64, 3), (5, 256, 64, 128), (77, 257, 136, 17), (129, 513, 200, 64), (256, 640, 264, 33), (257, 1024, 96, 32),
    (300, 5003, 384, 100), (700, 1500, 896, 5), (3000, 2000, 1800, 4), (60, 32000, 384, 64), (40, 3, 64, 10), (512, 700, 64, 20), (5000, 300, 64, 7),
])
@pytest.mark.parametrize("teacher", [torch.float32, torch.bfloat16])
def test_teacher(rows, vocab, dim, top, teacher):
    check(Problem(rows, vocab, dim, top=top, seed=rows, teacher=teacher, scale=0.5))


@pytest.mark.parametrize("top", [0, 9])
@pytest.mark.parametrize("scale", [0.1, 1.0, 3.0])
def test_scale_and_narrow_indices(top, scale):
    check(Problem(200, 900, 128, top=top, scale=scale, index=torch.int32, seed=4))


@pytest.mark.parametrize("top", [0, 6])
def test_several_pieces_of_the_vocabulary(top):
    """More dz than a piece holds: 16384 rows x 8960 words in two pieces of 18 and 17 tiles."""
    check(Problem(16384, 8960, 64, top=top, seed=5, left_out=0.02))


def test_many_splits_and_pieces():
    """Few row tiles against a long vocabulary: dx's sums in many parts."""
    check(Problem(20, 40000, 64, seed=6))


@pytest.mark.parametrize("top", [0, 4])
def test_large_logits(top):
    """Scores up to hundreds: the largest is taken out of every exponential."""
    check(Problem(100, 700, 64, top=top, spread=40.0, seed=8))


@pytest.mark.parametrize("top", [0, 4])
def test_one_gradient_for_all_rows(top):
    p = Problem(150, 400, 64, top=top, seed=9)
    check(p, dloss=torch.full((), 0.25, device="cuda").expand(150))
    every_other = torch.randn(300, device="cuda")[::2]
    check(p, dloss=every_other)


@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("rows,vocab", [(200, 700), (900, 700), (6000, 5000)])
def test_rows_that_take_no_part(top, rows, vocab):
    """NaN and infinities in what is left out change nothing; their own results are zeros."""
    p = Problem(rows, vocab, 136, top=top, seed=10, left_out=0.5)
    want = check(p)
    out = p.weights()[1].sum(1) == 0
    assert 0 < int(out.sum()) < rows
    p.x[out] = torch.tensor([math.nan, math.inf, -math.inf, 1e38], device="cuda").bfloat16().repeat(34)
    p.dloss[out] = math.nan
    if top:
        p.teacher[(p.index < 0) | (p.index >= p.vocab)] = math.nan
    plan = plan_of(p)
    loss, lse = forward(plan, p)
    lse_in = torch.where(out, torch.full_like(lse, math.nan), lse)
    dx, dw = backward(plan, p, lse_in)
    assert all(torch.equal(x, y) for x, y in zip((loss, lse, dx, dw), want))
    assert not loss[out].any() and not lse[out].any() and not dx[out].any()


@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("rows,vocab", [(30, 700), (600, 700), (6000, 12000)])
def test_no_row_takes_part(top, rows, vocab):
    p = Problem(rows, vocab, 136, top=top, left_out=2.0)
    p.x.fill_(math.nan)
    plan = plan_of(p)
    loss, lse = forward(plan, p)
    dx, dw = backward(plan, p, lse)
    assert not any(bool(t.any()) for t in (loss, lse, dx, dw))


@pytest.mark.parametrize("top", [0, 5])
def test_no_rows(top):
    p = Problem(0, 700, 136, top=top)
    plan = plan_of(p)
    loss, lse = forward(plan, p)
    dx, dw = backward(plan, p, lse)
    assert dx.shape == (0, 136) and not bool(dw.any())


def test_teacher_rows_of_one_kind():
    """All entries the same word; all logits -inf; an infinite and a NaN logit."""
    p = Problem(6, 300, 64, top=4, left_out=0.0)
    p.index[:] = torch.arange(4, device="cuda")
    p.index[1] = 17
    p.teacher[:] = 1.0
    p.teacher[2] = -math.inf
    p.teacher[3] = torch.finfo(torch.float32).min
    p.teacher[4, 0], p.teacher[5, 1] = math.inf, math.nan
    loss, lse = forward(plan_of(p), p)
    assert bool(torch.isnan(loss[4:]).all()) and float(loss[2]) == 0.0 and float(lse[2]) == 0.0
    p.teacher[4, 0] = p.teacher[5, 1] = 1.0
    check(p)


@pytest.mark.parametrize("teacher", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [0.25, 1.0, 4.0])
def test_teacher_masked_by_the_lowest_value(teacher, scale):
    """Entries at the type's lowest value beside ordinary ones, and beside its highest: no weight, and no NaN."""
    p = Problem(8, 300, 64, top=5, left_out=0.0, teacher=teacher, scale=scale)
    p.index[:] = torch.arange(5, device="cuda") * 50
    p.teacher[:] = torch.randn(8, 5, device="cuda").to(teacher)
    info = torch.finfo(teacher)
    p.teacher[:4, 1:3] = info.min
    p.teacher[4:6, 0], p.teacher[4:6, 1] = info.max, info.min
    check(p)


def test_a_nan_reaches_its_row_only():
    p = Problem(200, 300, 64, left_out=0.0)
    want = check(p)
    p.x[77, 3] = math.nan
    plan = plan_of(p)
    loss, lse = forward(plan, p)
    dx, dw = backward(plan, p, torch.where(torch.isnan(lse), want[1], lse))
    rest = torch.arange(200, device="cuda") != 77
    assert torch.equal(loss[rest], want[0][rest]) and bool(torch.isnan(loss[77]))
    assert torch.equal(dx[rest], want[2][rest]) and bool(torch.isnan(dx[77]).all()) and bool(torch.isnan(dw).all())


@pytest.mark.parametrize("top", [0, 5])
def test_steps(top):
    """Operands and results as parts of something larger, which stays as it was."""
    p = Problem(130, 500, 72, top=top, seed=11)
    want = check(p)
    wide_x, wide_w = torch.full((130, 200), 3.0, device="cuda").bfloat16(), torch.full((510, 104), 3.0, device="cuda").bfloat16()
    wide_x[:, 8:80], wide_w[5:505, 16:88] = p.x, p.w
    x, w = wide_x[:, 8:80], wide_w[5:505, 16:88]
    big_dx, big_dw = torch.full((140, 96), 9.0, device="cuda").bfloat16(), torch.full((510, 80), 9.0, device="cuda").bfloat16()
    plan = plan_of(p)
    loss, lse = forward(plan, p, x=x, w=w)
    dx, dw = backward(plan, p, lse, x=x, w=w, dx=big_dx[4:134, 16:88], dw=big_dw[1:501, :72])
    assert all(torch.equal(a, b) for a, b in zip((loss, lse, dx, dw), want))
    edge = big_dx.clone(); edge[4:134, 16:88] = 9.0
    assert bool((edge == 9.0).all())
    edge = big_dw.clone(); edge[1:501, :72] = 9.0
    assert bool((edge == 9.0).all())


def test_one_row_for_all():
    """x with a step of zero."""
    p = Problem(50, 300, 64, left_out=0.0)
    p.x[:] = p.x[:1].clone()
    want = check(p)
    x = p.x[:1].expand(50, 64)
    plan = plan_of(p)
    loss, lse = forward(plan, p, x=x)
    dx, dw = backward(plan, p, lse, x=x)
    assert torch.equal(loss, want[0])
    p.solve(lse=lse, gathered=True)
    assert off_by(dx, p.dx, p.dx_off) <= 1 and off_by(dw, p.dw, p.dw_off) <= 1


@pytest.mark.parametrize("rows", [1, 2, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("top", [0, 3])
def test_few_rows_lose_no_precision_on_the_way(rows, top):
    """A word's gradient is often one row's: dz is not rounded to bf16 there, only the results are."""
    check(Problem(rows, 1000, 200, top=top, seed=rows, left_out=0.1))


@pytest.mark.parametrize("top", [0, 20])
@pytest.mark.parametrize("rows", [90, 700, 5000])
def test_the_same_bits_every_time_on_any_stream_and_in_a_graph(top, rows):
    p = Problem(rows, 3000, 264, top=top, seed=12)
    plan = plan_of(p)
    loss, lse = forward(plan, p)
    want = (loss, lse) + backward(plan, p, lse)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        loss, lse = forward(plan, p)
        got = (loss, lse) + backward(plan, p, lse)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    dx, dw = torch.zeros_like(p.x), torch.zeros_like(p.w)
    with torch.cuda.graph(graph):
        loss, lse = forward(plan, p)
        backward(plan, p, lse, dx=dx, dw=dw)
    for _ in range(3):
        for t in (loss, lse, dx, dw):
            t.fill_(5.0)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip((loss, lse, dx, dw), want))
    # other rows take part when the graph runs again
    q = Problem(rows, 3000, 264, top=top, seed=13, left_out=0.8)
    for a, b in ((p.x, q.x), (p.w, q.w), (p.index, q.index), (p.dloss, q.dloss)) + (((p.teacher, q.teacher),) if top else ()):
        a.copy_(b)
    graph.replay()
    q.solve(lse=lse)
    assert off_by(loss, q.loss, q.loss_off) <= 1 and off_by(dx, q.dx, q.dx_off) <= 1 and off_by(dw, q.dw, q.dw_off) <= 1


@pytest.mark.parametrize("top", [0, 3])
def test_autograd(top):
    """The mean over the rows that count, against 64-bit autograd and against differences."""
    p = Problem(90, 200, 64, top=top, seed=14)
    x, w = p.x.clone().requires_grad_(True), p.w.clone().requires_grad_(True)
    plan = plan_of(p)
    losses = distill(plan, x, w, p.index, p.teacher) if top else cross_entropy(plan, x, w, p.index)
    at, t = p.weights()
    n = int((t.sum(1) > 0).sum())
    dx, dw = torch.autograd.grad(losses.sum() / n, (x, w))
    p.solve(lse=forward(plan, p)[1], dloss=torch.full((90,), 1 / n, device="cuda"))
    assert off_by(dx, p.dx, p.dx_off) <= 1 and off_by(dw, p.dw, p.dw_off) <= 1

    def total(x, w):
        z = p.scale * (x @ w.T)
        return ((torch.xlogy(t, t) - t * z.gather(1, at)).sum(1) + t.sum(1) * torch.logsumexp(z, 1)).sum() / n
    xd, wd = p.x.double(), p.w.double()
    for _ in range(3):
        ex, ew = torch.randn_like(xd), torch.randn_like(wd)
        h = 1e-5
        slope = (total(xd + h * ex, wd + h * ew) - total(xd - h * ex, wd - h * ew)) / (2 * h)
        got = (dx.double() * ex).sum() + (dw.double() * ew).sum()
        bound = (p.dx_off * ex.abs()).sum() + (p.dw_off * ew.abs()).sum() + 1e-6
        assert abs(float(got - slope)) <= float(bound)


def test_second_derivatives_are_refused():
    p = Problem(10, 30, 16)
    x, w = p.x.clone().requires_grad_(True), p.w.clone().requires_grad_(True)
    loss = cross_entropy(plan_of(p), x, w, p.index).sum()
    first = torch.autograd.grad(loss, (x, w), create_graph=True)
    with pytest.raises(RuntimeError):
        sum((g.float() ** 2).sum() for g in first).backward()


@pytest.mark.parametrize("rows,vocab,dim,top", [(300000, 700, 64, 0), (200001, 300, 32, 2), (50, 600007, 64, 0), (50, 600007, 64, 3)])
def test_many_rows_and_long_vocabularies(rows, vocab, dim, top):
    check(Problem(rows, vocab, dim, top=top, seed=20, left_out=0.01))


@pytest.mark.parametrize("top", [0, 3])
def test_offsets_beyond_32_bits(top):
    """Rows of every operand 2^20 + 8 elements apart: the last ones lie more than 2^31 elements behind the first."""
    rows, vocab, dim = 2200, 2100, 64
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 20 GB")
    p = Problem(rows, vocab, dim, top=top, seed=21)
    want = check(p)
    step = (1 << 20) + 8
    apart = lambda n: torch.empty(n * step, dtype=torch.bfloat16, device="cuda").view(n, step)[:, 8:8 + dim]  # noqa: E731
    x, w, dx, dw = apart(rows), apart(vocab), apart(rows), apart(vocab)
    x.copy_(p.x)
    w.copy_(p.w)
    plan = plan_of(p)
    loss, lse = forward(plan, p, x=x, w=w)
    backward(plan, p, lse, x=x, w=w, dx=dx, dw=dw)
    assert all(torch.equal(a, b) for a, b in zip((loss, lse, dx, dw), want))
