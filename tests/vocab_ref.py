"""The losses over a vocabulary and their gradients in 64 bits, with bounds on what the kernels' roundings may do."""
import math

import torch

HALF_BF16 = 2.0 ** -8       # a rounding to bf16, relative
EPS = 2.0 ** -23            # a step of binary32, relative


class Problem:
    """Inputs on the device, their 64-bit forms and results.  `labels`: [rows] targets; with `teacher` [rows, top] indices."""

    def __init__(self, rows, vocab, dim, top=0, scale=1.0, seed=0, index=torch.int64, teacher=torch.float32, left_out=0.25, spread=1.0,
                 device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.vocab, self.dim, self.top, self.scale = rows, vocab, dim, top, scale
        self.x = (spread * torch.randn(rows, dim, generator=g)).bfloat16().to(device)
        self.w = (torch.randn(vocab, dim, generator=g) * 2 / math.sqrt(dim)).bfloat16().to(device)
        out = torch.rand(rows, generator=g) < left_out
        if top:
            at = torch.randint(vocab, (rows, top), generator=g)          # one word may come several times
            at[torch.rand(rows, top, generator=g) < 0.1] = -1
            at[torch.rand(rows, top, generator=g) < 0.1] = vocab
            at[out] = -7
            t = 3 * torch.randn(rows, top, generator=g)
            t[torch.rand(rows, top, generator=g) < 0.1] = -math.inf
            self.index, self.teacher = at.to(index).to(device), t.to(teacher).to(device)
        else:
            at = torch.randint(vocab, (rows,), generator=g)
            at[out] = torch.tensor([-100, -1, vocab, vocab + 5])[torch.randint(4, (int(out.sum()),), generator=g)]
            self.index, self.teacher = at.to(index).to(device), None
        self.dloss = (torch.randn(rows, generator=g) / max(1, rows)).to(device)

    def weights(self):
        """(indices, 64-bit weights) [rows, max(1, top)]; entries that take no part have weight 0."""
        at = self.index.long().view(self.rows, -1)
        ok = (at >= 0) & (at < self.vocab)
        if self.teacher is None:
            return at.clamp(0, self.vocab - 1), ok.double()
        t = self.teacher.double()
        ok &= t != -math.inf
        t = torch.where(ok, self.scale * t, -math.inf)
        top = t.amax(1, keepdim=True)
        t = torch.where(ok, (t - torch.where(top == -math.inf, 0.0, top)).exp(), 0.0)
        return at.clamp(0, self.vocab - 1), t / t.sum(1, keepdim=True).clamp(min=1e-300)

    def solve(self, lse=None, dloss=None, gathered=False):
        """loss, lse, dx, dw and a bound on the error of each.  lse, dloss: what the backward pass is given (else its own).
        Up to 64 rows, unless they are gathered, dz goes in two bf16 parts: what is left is off by a rounding of a rounding."""
        at, t = self.weights()
        used = t.sum(1) > 0
        x, w = torch.where(used[:, None], self.x.double(), 0.0), self.w.double()
        z = self.scale * (x @ w.T)
        # products of bf16 are exact in binary32; each of `dim` additions is off by at most a step of the running sum
        z_off = self.scale * self.dim * EPS * (x.abs() @ w.abs().T).amax(1)
        s = torch.logsumexp(z, 1)
        self.lse = torch.where(used, s, 0.0)
        self.loss = torch.where(used, (torch.xlogy(t, t) + t * (s[:, None] - z.gather(1, at))).sum(1), 0.0)
        top = z.abs().amax(1)
        # the exponent's two roundings, the exponential's 2 steps, a sum of 128 in each part of a tile and of the parts
        self.lse_off = z_off + (2 * top + 2 + 64 + self.vocab / 1024 + 16) * EPS + s.abs() * EPS
        entropy = torch.xlogy(t, t).abs().sum(1)
        self.loss_off = 2 * self.lse_off + (entropy + 4 * top + self.top) * EPS + self.loss.abs() * EPS
        lse = torch.where(used, (self.lse if lse is None else lse.double()), 0.0)
        dloss = torch.where(used, (self.dloss if dloss is None else dloss).double(), 0.0)
        p = torch.where(used[:, None], torch.exp(z - lse[:, None]), 0.0)
        both = p.scatter_add(1, at, t)
        dz = p.scatter_add(1, at, -t) * (self.scale * dloss)[:, None]
        p_off = z_off + (2 * top + 4 + lse.abs()) * EPS
        dz_off = (HALF_BF16 if gathered or self.rows > 64 else HALF_BF16 ** 2) * dz.abs() + (self.scale * dloss.abs() * (p_off + (4 + self.top) * EPS))[:, None] * both
        self.dx, self.dw = dz @ w, dz.T @ x
        self.dx_off = dz_off @ w.abs() + self.vocab * EPS * (dz.abs() @ w.abs()) + HALF_BF16 * self.dx.abs() + 1e-30
        self.dw_off = dz_off.T @ x.abs() + self.rows * EPS * (dz.abs().T @ x.abs()) + HALF_BF16 * self.dw.abs() + 1e-30
        # a bound's own roundings of second order
        for name in ("lse", "loss", "dx", "dw"):
            setattr(self, name + "_off", 1.02 * getattr(self, name + "_off"))
        return self


def off_by(got, want, bound):
    """Largest error as a share of its bound; NaN counts as infinite."""
    share = (got.double() - want).abs() / bound.clamp(min=1e-300)
    return float(torch.nan_to_num(share, nan=math.inf).max()) if share.numel() else 0.0
