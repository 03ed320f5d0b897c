"""A small language model trained by asynchronous Local-SGD workers, end to end on one GPU.

The workers' inner step is the library's: attention with a learned relative position bias (forward and backward), the
gradients' global norm and clipping into the flat vector, AdamW on it; and so is the server's: arrivals with Delayed
Nesterov, DyLU step counts, the learning-rate schedule and the scheduler.  Embedding, layer norms, the linear maps and the
loss are plain PyTorch on the worker's bf16 replica.

The data is made here: every token repeats the one LAG places earlier, except for a share of random ones that differs from
shard to shard, and sequences end at different lengths.  Nothing but attention can know the earlier token, and nothing but
its position can tell which one it is.

    python -m paper_2401_09135_b200.lm
"""
from __future__ import annotations

import argparse
import math

import torch
import torch.nn.functional as F

from . import binding as B
from . import synth
from .attention import attend

VOCAB, WIDTH, HEADS, LAYERS, FF, BUCKETS = 64, 64, 2, 2, 128, 16
LENGTH, LAG, BATCH = 64, 5, 16


def tensors():
    """Parameters in flat order; the bias table is one more vector that is not weight-decayed."""
    T = synth.Tensor
    t = [T("tok_emb", VOCAB * WIDTH, True, "matrix"), T("bias_table", HEADS * BUCKETS, False, "bias")]
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

    def __init__(self, offsets, device, batch=BATCH):
        self.names, self.device = [t.name for t in tensors()], device
        self.offsets, self.sizes = offsets, [t.numel for t in tensors()]
        self.plan = B.Attention(batch, LENGTH, LENGTH, HEADS, HEADS, WIDTH // HEADS, causal=True, buckets=BUCKETS,
                                max_distance=32, table_dtype=torch.bfloat16, device=device.index)

    def loss(self, p, tokens, lengths):
        """Mean cross-entropy over the valid positions that have something to repeat; p: name -> tensor."""
        x = F.embedding(tokens[:, :-1], p["tok_emb"].view(VOCAB, WIDTH))
        b = x.shape[0]
        for l in range(LAYERS):
            h = F.layer_norm(x, (WIDTH,), p[f"l{l}.ln1.g"], p[f"l{l}.ln1.b"])
            q, k, v = (h @ p[f"l{l}.w_qkv"].view(WIDTH, 3 * WIDTH)).view(b, LENGTH, 3, HEADS, WIDTH // HEADS).unbind(2)
            a = attend(self.plan, q, k, v, p["bias_table"].view(HEADS, BUCKETS), lengths)
            x = x + a.reshape(b, LENGTH, WIDTH) @ p[f"l{l}.wo"].view(WIDTH, WIDTH)
            h = F.layer_norm(x, (WIDTH,), p[f"l{l}.ln2.g"], p[f"l{l}.ln2.b"])
            x = x + F.gelu(h @ p[f"l{l}.w_ff1"].view(WIDTH, FF)) @ p[f"l{l}.w_ff2"].view(FF, WIDTH)
        x = F.layer_norm(x, (WIDTH,), p["lnf.g"], p["lnf.b"])
        logits = (x @ p["tok_emb"].view(VOCAB, WIDTH).t()).float()
        at = torch.arange(LENGTH, device=tokens.device)
        use = (at >= LAG - 1) & (at < lengths[:, None])
        return F.cross_entropy(logits[use], tokens[:, 1:][use])

    def parameters(self, flat):
        return {n: flat[o:o + s] for n, o, s in zip(self.names, self.offsets, self.sizes)}

    def gradients(self, replica, tokens, lengths):
        """(loss, one bf16 gradient per tensor) at the replica's bit patterns."""
        leaves = {n: t.detach().requires_grad_(True) for n, t in self.parameters(replica.view(torch.bfloat16)).items()}
        loss = self.loss(leaves, tokens, lengths)
        return loss.detach(), list(torch.autograd.grad(loss, list(leaves.values())))


def theta0(P, offsets, seed):
    g = torch.Generator().manual_seed(seed)
    th = torch.zeros(P)
    for t, o in zip(tensors(), offsets):
        if t.kind == "matrix":
            th[o:o + t.numel] = torch.randn(t.numel, generator=g) * (0.5 if t.name == "tok_emb" else 1.0) / math.sqrt(WIDTH)
        elif t.kind == "gain":
            th[o:o + t.numel] = 1.0
    return th


def run(speeds=(1.0, 1.5, 2.0, 3.0), N=4, outer_lr=0.7, beta=0.9, H=20, tau_grace=0.5, total_local_steps=2000, max_norm=1.0,
        lr_max=3e-3, lr_min=3e-4, warmup=20, seed=7, device=0, log_every=0):
    """Asynchronous Local-SGD with DyLU.  Returns (validation loss before, after, server updates, share of steps clipped,
    final theta as a CPU tensor)."""
    torch.cuda.set_device(device)
    dev = torch.device("cuda", device)
    W = len(speeds)
    ctx = B.Context(tensors(), W, N, beta, outer_lr, adam=(0.9, 0.95, 1e-8, 0.1), align_elems=8, device=device)
    model = Model(ctx.offsets, dev)
    ctx.alsgd_set_global(theta0(ctx.P, ctx.offsets, seed).numpy())
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
        for _ in range(steps[w]):
            replica = ctx.alsgd_worker_state_ptrs(w)["replica"]
            _, grads = model.gradients(replica, *batch_of(w, w, life[w], seed, dev))
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
    if B.alsgd_attn_status(device):
        raise RuntimeError("a wait inside the attention kernels ran out")
    return before, after, updates, share, theta.cpu()


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=2000)
    args = ap.parse_args()
    before, after, updates, share, _ = run(total_local_steps=args.steps, log_every=20)
    print(f"validation loss {before:.4f} -> {after:.4f} (chance {math.log(VOCAB):.4f}) after {updates} server updates; "
          f"{100 * share:.0f} % of the inner steps were clipped")


if __name__ == "__main__":
    main()
