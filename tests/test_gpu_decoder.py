"""Rotary positions, attention, the loss over the vocabulary and its distillation together, as a worker's step runs them."""
import math

import pytest
import torch

from paper_2401_09135_b200 import binding as B
from paper_2401_09135_b200 import lm, synth
from paper_2401_09135_b200.attention import attend
from paper_2401_09135_b200.rotary import rotate
from paper_2401_09135_b200.vocab import cross_entropy, distill

pytestmark = pytest.mark.gpu


def turned(x):
    """Rotary positions in 64 bits, halves apart."""
    n, d = x.shape[1], x.shape[3]
    f = 10000.0 ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
    t = torch.arange(n, device=x.device)[:, None] * f
    cos, sin = t.cos()[:, None], t.sin()[:, None]
    a, b = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def attention(q, k, v, lengths):
    x = torch.einsum("bihd,bjhd->bhij", q, k) * q.shape[-1] ** -0.5
    j = torch.arange(k.shape[1], device=q.device)
    off = (j[None, :] > j[:, None])[None] | (j >= lengths[:, None])[:, None]
    return torch.einsum("bhij,bjhd->bihd", torch.softmax(x.masked_fill(off[:, None], -math.inf), -1), v)


@pytest.mark.parametrize("teacher", [False, True])
def test_a_decoder_layer_from_positions_to_the_loss(teacher):
    """rotate, attend and either loss in one graph against 64-bit autograd.  Every operator rounds its results to bf16 (2^-8 each,
    half a step) and its gradients' operands once more: with three operators on the way, norms agree to 8 roundings."""
    b, n, h, d, vocab, top = 2, 150, 4, 64, 1000, 6
    g = torch.Generator(device="cuda").manual_seed(0)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    qkv, w = rnd(b, n, 3, h, d), (rnd(vocab, h * d) * (2 / math.sqrt(h * d))).bfloat16()
    lengths = torch.tensor([150, 88], dtype=torch.int32, device="cuda")
    use = torch.arange(n, device="cuda") < lengths[:, None]
    words = torch.randint(vocab, (b, n, top), generator=g, device="cuda").masked_fill(~use[..., None], -100)
    logits = torch.randn(b, n, top, generator=g, device="cuda")

    def total(qkv, w, own):
        q, k, v = qkv.unbind(2)
        if own:
            a = attend(B.Attention(b, n, n, h, h, d), *rotate(B.Rotary(b, n, h, h, d), q, k), v, None, lengths).reshape(b * n, h * d)
            if teacher:
                losses = distill(B.VocabLoss(b * n, vocab, h * d, top=top), a, w, words.view(-1, top), logits.view(-1, top))
            else:
                losses = cross_entropy(B.VocabLoss(b * n, vocab, h * d), a, w, words[..., 0].reshape(-1).contiguous())
            return losses.sum() / use.sum()
        a = attention(turned(q), turned(k), v, lengths).reshape(b * n, h * d)
        log_p = torch.log_softmax(a @ w.T, -1)
        k = top if teacher else 1
        t = torch.softmax(logits.double().view(-1, top), -1) if teacher else torch.ones(1, 1, device="cuda", dtype=torch.float64)
        at = words.view(-1, top)[:, :k].clamp(min=0)
        return ((t * (t.log() - log_p.gather(1, at))).sum(1) * use.view(-1)).sum() / use.sum()

    leaves = [t.clone().requires_grad_(True) for t in (qkv, w)]
    wide = [t.double().requires_grad_(True) for t in (qkv, w)]
    mine, exact = total(*leaves, True), total(*wide, False)
    assert abs(float(mine.detach()) - float(exact.detach())) <= 2.0 ** -8 * abs(float(exact.detach()))
    for x, y in zip(torch.autograd.grad(mine, leaves), torch.autograd.grad(exact, wide)):
        assert float((x.double() - y).norm()) <= 8 * 2.0 ** -8 * float(y.norm())


@pytest.mark.parametrize("rotary", [False, True])
def test_the_models_loss_without_its_logits_has_the_same_gradients(rotary):
    """Against the model's own loss in PyTorch on the same replica.  Both round in bf16 on the way (the plain one its logits as well,
    2^-8 of at most about 8 each): gradients agree to 16 roundings in norm, tensor by tensor."""
    dev = torch.device("cuda", 0)
    P, offs = B.alsgd_layout_size(lm.tensors(rotary), 8)
    replica = lm.theta0(P, offs, 3, rotary).bfloat16().to(dev).view(torch.int16)
    tokens, lengths = lm.batch_of(1, 0, 0, 5, dev)
    plain, own = (lm.Model(offs, dev, rotary=rotary, vocab_loss=v) for v in (False, True))
    (la, ga), (lb, gb) = plain.gradients(replica, tokens, lengths), own.gradients(replica, tokens, lengths)
    assert abs(float(la) - float(lb)) <= 2.0 ** -7 * abs(float(la))
    for name, x, y in zip(plain.names, ga, gb):
        assert float((x.double() - y.double()).norm()) <= 16 * 2.0 ** -8 * float(x.double().norm()), name


def test_distillation_from_the_model_itself_pulls_nowhere_but_to_its_own_top():
    """With the worker's own replica as the teacher the distance is that of the top's softmax from the whole one, and the gradient
    of the sum is the loss's and the distance's."""
    dev = torch.device("cuda", 0)
    P, offs = B.alsgd_layout_size(lm.tensors(True), 8)
    replica = lm.theta0(P, offs, 4, True).bfloat16().to(dev).view(torch.int16)
    tokens, lengths = lm.batch_of(0, 0, 0, 6, dev)
    model = lm.Model(offs, dev, rotary=True, vocab_loss=True, distill_weight=0.5)
    teacher = model.highest_logits(model.parameters(replica.view(torch.bfloat16)), tokens, lengths)
    p = model.parameters(replica.view(torch.bfloat16))
    x = model.hidden(p, tokens, lengths).reshape(-1, lm.WIDTH)
    z = x.double() @ p["tok_emb"].view(lm.VOCAB, lm.WIDTH).double().T / lm.TEMPERATURE
    use = model.counted(lengths).reshape(-1)
    t = torch.softmax(teacher[1].double() / lm.TEMPERATURE, -1)
    want = ((t * (t.log() - torch.log_softmax(z, -1).gather(1, teacher[0].clamp(min=0)))).sum(1) * use).sum() / use.sum()
    with_it, _ = model.gradients(replica, tokens, lengths, replica)
    without, _ = model.gradients(replica, tokens, lengths)
    got = float(with_it - without) / (0.5 * lm.TEMPERATURE ** 2)
    # the two means are binary32 sums of binary32 losses
    assert abs(got - float(want)) <= 1e-4 * max(1.0, abs(float(want)))


@pytest.mark.parametrize("options", [dict(rotary=True), dict(vocab_loss=True), dict(rotary=True, vocab_loss=True, distill_weight=0.3)])
def test_training_runs_and_the_same_seed_gives_the_same_model(options):
    a, b = (lm.run(total_local_steps=80, **options) for _ in range(2))
    assert a[2] > 0 and bool(torch.isfinite(a[4]).all()) and math.isfinite(a[1])
    assert a[1] == b[1] and torch.equal(a[4], b[4])


def test_the_papers_vocabulary_with_a_clipped_step():
    """Gradients of the 32 000-word embedding go straight into the flat vector of a worker."""
    rows, vocab, dim = 200, 32000, 384
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, dim, generator=g, device="cuda").bfloat16().requires_grad_(True)
    w = (0.02 * torch.randn(vocab, dim, generator=g, device="cuda")).bfloat16().requires_grad_(True)
    target = torch.randint(vocab, (rows,), generator=g, device="cuda")
    dw, = torch.autograd.grad(cross_entropy(B.VocabLoss(rows, vocab, dim), x, w, target).mean(), w)
    ctx = B.Context([synth.Tensor("tok_emb", vocab * dim, True, "matrix")], 1, 1, 0.9, 0.7)
    flat, stats = torch.zeros(ctx.P, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, device="cuda")
    B.GradClip([vocab * dim], ctx.offsets, [torch.bfloat16], torch.bfloat16).alsgd_clip_grads([dw], 0.1, flat, stats)
    assert abs(float(stats[0]) - float(dw.double().norm())) <= 1e-5 * float(stats[0])
    ctx.alsgd_set_global(w.detach().float().flatten())
    ctx.alsgd_pull(0)
    ctx.alsgd_inner_adamw_bf16(0, flat, 1, 1e-3)
    ctx.alsgd_sync()
    assert bool(torch.isfinite(ctx.alsgd_worker_state_ptrs(0)["p"]).all())
    ctx.close()


def test_calls_on_several_streams_at_once():
    """Plans of their own, streams of their own: losses, attention and rotary positions side by side give the bits that they give
    one after the other."""
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
    jobs = []
    for rows, vocab, dim in ((700, 3000, 264), (90, 5000, 128), (2000, 1000, 64)):
        x, w, target = rnd(rows, dim), rnd(vocab, dim) * 0.1, torch.randint(-1, vocab, (rows,), generator=g, device="cuda")
        plan, dloss = B.VocabLoss(rows, vocab, dim), torch.full((rows,), 1 / rows, device="cuda")

        def loss(x=x, w=w, target=target, plan=plan, dloss=dloss, rows=rows):
            out = [torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(w)]
            plan.alsgd_xent_fwd(x, w, target, *out[:2])
            plan.alsgd_xent_bwd(x, w, target, out[1], dloss, *out[2:])
            return out
        jobs.append(loss)
    q, k, v = (rnd(4, 500, 4, 64) for _ in range(3))
    attention_plan, rotary = B.Attention(4, 500, 500, 4, 4, 64), B.Rotary(4, 500, 4, 4, 64)

    def attends():
        out = [torch.empty_like(q) for _ in range(3)] + [torch.empty(4, 4, 500, device="cuda")]
        rotary.alsgd_rope(q, k, *out[:2])
        attention_plan.alsgd_attn_fwd(out[0], out[1], v, out[2], out[3])
        return out
    jobs.append(attends)
    want = [j() for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(10):
        got = []
        for s, j in zip(streams, jobs):
            with torch.cuda.stream(s):
                got.append(j())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
    assert B.alsgd_vocab_status() == 0 and B.alsgd_attn_status() == 0


@pytest.mark.parametrize("rows", [40, 300, 700])
def test_two_graphs_that_share_a_plan(rows):
    """Captured one after the other, replayed in any order on one stream."""
    g = torch.Generator(device="cuda").manual_seed(3)
    vocab, dim = 2000, 128
    plan, dloss = B.VocabLoss(rows, vocab, dim), torch.full((), 1 / rows, device="cuda").expand(rows)
    w = (0.1 * torch.randn(vocab, dim, generator=g, device="cuda")).bfloat16()
    graphs, outs, want, steps = [], [], [], []     # steps: a graph reads its operands where they were
    for i in range(2):
        x, target = torch.randn(rows, dim, generator=g, device="cuda").bfloat16(), torch.randint(-1, vocab, (rows,), generator=g, device="cuda")
        out = [torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros_like(x), torch.zeros_like(w)]

        def step(x=x, target=target, out=out):
            plan.alsgd_xent_fwd(x, w, target, *out[:2])
            plan.alsgd_xent_bwd(x, w, target, out[1], dloss, *out[2:])
        step()
        want.append([t.clone() for t in out])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        graphs.append(graph)
        outs.append(out)
        steps.append(step)
    for i in (0, 1, 1, 0, 1):
        for t in outs[i]:
            t.fill_(3.0)
        graphs[i].replay()
        assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i]))
