"""A small language model trained by asynchronous Local-SGD workers, end to end on one GPU.

The workers' inner step is the library's: attention with a learned relative position bias (forward and backward), the
gradients' global norm and clipping into the flat vector, AdamW on it; and so is the server's: arrivals with Delayed
Nesterov, DyLU step counts, the learning-rate schedule and the scheduler.  Embedding, layer norms, the linear maps and the
loss are plain PyTorch on the worker's bf16 replica.  On request positions are rotary in place of the learned bias, the loss
is the library's too (the logits are never kept), and workers are held near the model that they were dispatched with by
distillation from its highest logits.

The data is made here: every token repeats the one LAG places earlier, except for a share of random ones that differs from
shard to shard, and sequences end at different lengths.  Nothing but attention can know the earlier token, and nothing but
its position can tell which one it is.

    python -m paper_2401_09135_b200.lm [--rotary] [--vocab-loss] [--distill 0.3]
"""
from __future__ import annotations

import argparse
import math

import torch
import torch.nn.functional as F

from . import binding as B
from . import synth
from .attention import attend
from .rotary import rotate
from .vocab import cross_entropy, distill

VOCAB, WIDTH, HEADS, LAYERS, FF, BUCKETS = 64, 64, 2, 2, 128, 16
LENGTH, LAG, BATCH = 64, 5, 16
TEACHER_TOP, TEMPERATURE = 8, 2.0


def tensors(rotary=False):
    """Parameters in flat order; the bias table, without rotary positions, is one more vector that is not weight-decayed."""
    T = synth.Tensor
    t = [T("tok_emb", VOCAB * WIDTH, True, "matrix")] + ([] if rotary else [T("bias_table", HEADS * BUCKETS, False, "bias")])
    for l in range(LAYERS):
        t += [T(f"l{l}.ln1.g", WIDTH, False, "gain"), T(f"l{l}.ln1.b", WIDTH, False, "bias"),
              T(f"l{l}.w_qkv", WIDTH * 3 * WIDTH, True, "matrix"), T(f"l{l}.wo", WIDTH * WIDTH, True, "matrix"),
              T(f"l{l}.ln2.g", WIDTH, False, "gain"), T(f"l{l}.ln2.b", WIDTH, False, "bias"),
              T(f"l{l}.w_ff1", WIDTH * FF, True, "matrix"), T(f"l{l}.w_ff2", FF * WIDTH, True, "matrix")]
    return t + [T("lnf.g", WIDTH, False, "gain"), T("lnf.b", WIDTH, False, "bias")]


def batch_of(shard, worker, step, seed, device, batch=BATCH):
    """(tokens [batch, LENGTH + 1], valid lengths) of a worker's step; shard s replaces a share of 5 + 5 s % at random."""
    g = torch.Generator(device=device).manual_seed(seed * 1_000_003 + worker * 10_007 + step)
    first = torch.randint(VOCAB, (batch, LAG), generator=g, device=device)
    x = first.repeat(1, -(-(LENGTH + 1) // LAG))[:, :LENGTH + 1]
    noise = torch.rand(x.shape, generator=g, device=device) < 0.05 * (shard + 1)
    x = torch.where(noise, torch.randint(VOCAB, x.shape, generator=g, device=device), x)
    return x, torch.randint(LENGTH // 2, LENGTH + 1, (batch,), generator=g, device=device, dtype=torch.int32)


class Model:
    """Loss and gradients at a worker's bf16 replica."""

    def __init__(self, offsets, device, batch=BATCH, rotary=False, vocab_loss=False, distill_weight=0.0):
        ts = tensors(rotary)
        self.names, self.device = [t.name for t in ts], device
        self.offsets, self.sizes = offsets, [t.numel for t in ts]
        self.plan = B.Attention(batch, LENGTH, LENGTH, HEADS, HEADS, WIDTH // HEADS, causal=True, buckets=0 if rotary else BUCKETS,
                                max_distance=32, table_dtype=torch.bfloat16, device=device.index)
        self.rotary = B.Rotary(batch, LENGTH, HEADS, HEADS, WIDTH // HEADS, device=device.index) if rotary else None
        self.labels = B.VocabLoss(batch * LENGTH, VOCAB, WIDTH, device=device.index) if vocab_loss else None
        self.distill_weight = distill_weight
        self.teacher = B.VocabLoss(batch * LENGTH, VOCAB, WIDTH, top=TEACHER_TOP, scale=1 / TEMPERATURE,
                                   teacher_dtype=torch.bfloat16, device=device.index) if distill_weight else None

    def hidden(self, p, tokens, lengths):
        """What stands behind the last norm; p: name -> tensor."""
        x = F.embedding(tokens[:, :-1], p["tok_emb"].view(VOCAB, WIDTH))
        b = x.shape[0]
        for l in range(LAYERS):
            h = F.layer_norm(x, (WIDTH,), p[f"l{l}.ln1.g"], p[f"l{l}.ln1.b"])
            q, k, v = (h @ p[f"l{l}.w_qkv"].view(WIDTH, 3 * WIDTH)).view(b, LENGTH, 3, HEADS, WIDTH // HEADS).unbind(2)
            if self.rotary:
                a = attend(self.plan, *rotate(self.rotary, q, k), v, None, lengths)
            else:
                a = attend(self.plan, q, k, v, p["bias_table"].view(HEADS, BUCKETS), lengths)
            x = x + a.reshape(b, LENGTH, WIDTH) @ p[f"l{l}.wo"].view(WIDTH, WIDTH)
            h = F.layer_norm(x, (WIDTH,), p[f"l{l}.ln2.g"], p[f"l{l}.ln2.b"])
            x = x + F.gelu(h @ p[f"l{l}.w_ff1"].view(WIDTH, FF)) @ p[f"l{l}.w_ff2"].view(FF, WIDTH)
        return F.layer_norm(x, (WIDTH,), p["lnf.g"], p["lnf.b"])

    @staticmethod
    def counted(lengths):
        """Valid positions that have something to repeat."""
        at = torch.arange(LENGTH, device=lengths.device)
        return (at >= LAG - 1) & (at < lengths[:, None])

    def loss(self, p, tokens, lengths, teacher=None):
        """Mean cross-entropy over the positions that count, and its distance from a teacher's (words, logits)."""
        x, use, w = self.hidden(p, tokens, lengths), self.counted(lengths), p["tok_emb"].view(VOCAB, WIDTH)
        if self.labels:
            target = torch.where(use, tokens[:, 1:], -100).reshape(-1)
            loss = cross_entropy(self.labels, x.reshape(-1, WIDTH), w, target).sum() / use.sum()
        else:
            loss = F.cross_entropy((x @ w.t()).float()[use], tokens[:, 1:][use])
        if teacher is not None:
            apart = distill(self.teacher, x.reshape(-1, WIDTH), w, *teacher).sum() / use.sum()
            loss = loss + self.distill_weight * TEMPERATURE ** 2 * apart
        return loss

    def highest_logits(self, p, tokens, lengths):
        """A model's TEACHER_TOP words and logits at every position that counts; no words at the others."""
        with torch.no_grad():
            top = (self.hidden(p, tokens, lengths) @ p["tok_emb"].view(VOCAB, WIDTH).t()).topk(TEACHER_TOP)
            words = torch.where(self.counted(lengths)[..., None], top.indices, -1)
            return words.view(-1, TEACHER_TOP), top.values.view(-1, TEACHER_TOP)

    def parameters(self, flat):
        return {n: flat[o:o + s] for n, o, s in zip(self.names, self.offsets, self.sizes)}

    def gradients(self, replica, tokens, lengths, teacher=None):
        """(loss, one bf16 gradient per tensor) at the replica's bit patterns; teacher: bit patterns of another one."""
        leaves = {n: t.detach().requires_grad_(True) for n, t in self.parameters(replica.view(torch.bfloat16)).items()}
        if teacher is not None:
            teacher = self.highest_logits(self.parameters(teacher.view(torch.bfloat16)), tokens, lengths)
        loss = self.loss(leaves, tokens, lengths, teacher)
        return loss.detach(), list(torch.autograd.grad(loss, list(leaves.values())))


def theta0(P, offsets, seed, rotary=False):
    g = torch.Generator().manual_seed(seed)
    th = torch.zeros(P)
    for t, o in zip(tensors(rotary), offsets):
        if t.kind == "matrix":
            th[o:o + t.numel] = torch.randn(t.numel, generator=g) * (0.5 if t.name == "tok_emb" else 1.0) / math.sqrt(WIDTH)
        elif t.kind == "gain":
            th[o:o + t.numel] = 1.0
    return th


def run(speeds=(1.0, 1.5, 2.0, 3.0), N=4, outer_lr=0.7, beta=0.9, H=20, tau_grace=0.5, total_local_steps=2000, max_norm=1.0,
        lr_max=3e-3, lr_min=3e-4, warmup=20, seed=7, device=0, log_every=0, rotary=False, vocab_loss=False, distill_weight=0.0):
    """Asynchronous Local-SGD with DyLU.  Returns (validation loss before, after, server updates, share of steps clipped,
    final theta as a CPU tensor)."""
    torch.cuda.set_device(device)
    dev = torch.device("cuda", device)
    W = len(speeds)
    ctx = B.Context(tensors(rotary), W, N, beta, outer_lr, adam=(0.9, 0.95, 1e-8, 0.1), align_elems=8, device=device)
    model = Model(ctx.offsets, dev, rotary=rotary, vocab_loss=vocab_loss, distill_weight=distill_weight)
    ctx.alsgd_set_global(theta0(ctx.P, ctx.offsets, seed, rotary).numpy())
    clip = B.GradClip(model.sizes, ctx.offsets, [torch.bfloat16] * len(model.sizes), torch.bfloat16, device=device)
    flat, stats = torch.zeros(ctx.P, dtype=torch.bfloat16, device=dev), torch.zeros(2, device=dev)
    clipped = torch.zeros((), device=dev)
    steps = B.alsgd_dylu_steps(speeds, H)
    sched = B.Scheduler(W, tau_grace, t_max=total_local_steps)
    per_worker = total_local_steps // W
    life = [0] * W

    val = batch_of(0, W, 0, seed, dev)

    def validation():
        theta = ctx.alsgd_state_ptrs()[0].bfloat16()
        with torch.no_grad():
            return float(model.loss(model.parameters(theta), *val))

    def train(w):
        # the model that the worker was dispatched with
        teacher = ctx.alsgd_worker_state_ptrs(w)["replica"].clone() if distill_weight else None
        for _ in range(steps[w]):
            replica = ctx.alsgd_worker_state_ptrs(w)["replica"]
            _, grads = model.gradients(replica, *batch_of(w, w, life[w], seed, dev), teacher)
            clip.alsgd_clip_grads(grads, max_norm, flat, stats)
            clipped.add_(stats[1] < 1.0)
            life[w] += 1
            ctx.alsgd_inner_adamw_bf16(w, flat, life[w], B.alsgd_lr_at(lr_max, lr_min, warmup, per_worker, life[w]))
        sched.dispatch(w, steps[w] / speeds[w], steps[w])

    before = validation()
    for w in range(W):
        ctx.alsgd_pull(w)
    for w in range(W):
        train(w)
    updates = 0
    while True:
        ids, _, _ = sched.next_batch()
        if not ids:
            break
        ctx.alsgd_arrive(ids, B.ARRIVE_RESEED, want_info=False)
        updates += len(ids)
        if log_every and updates % log_every < len(ids):
            print(f"  update {updates}: val loss {validation():.4f}")
        for w in ids:
            train(w)
    after = validation()
    theta = ctx.alsgd_state_ptrs()[0].clone()
    ctx.alsgd_sync()
    share = float(clipped) / max(1, sum(life))
    ctx.close()
    if B.alsgd_attn_status(device) or B.alsgd_vocab_status(device):
        raise RuntimeError("a wait inside the kernels ran out")
    return before, after, updates, share, theta.cpu()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=2000)
    ap.add_argument("--rotary", action="store_true", help="rotary positions in place of the learned bias")
    ap.add_argument("--vocab-loss", action="store_true", help="the loss without its logits")
    ap.add_argument("--distill", type=float, default=0.0, help="weight of the distance from the model that a worker was dispatched with")
    args = ap.parse_args()
    before, after, updates, share, _ = run(total_local_steps=args.steps, log_every=20, rotary=args.rotary, vocab_loss=args.vocab_loss,
                                           distill_weight=args.distill)
    print(f"validation loss {before:.4f} -> {after:.4f} (chance {math.log(VOCAB):.4f}) after {updates} server updates; "
          f"{100 * share:.0f} % of the inner steps were clipped")


if __name__ == "__main__":
    main()
