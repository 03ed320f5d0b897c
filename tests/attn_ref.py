"""Attention with a bucketed relative position bias and its gradients, written from the formulas in 64 bits, one head
of one sequence at a time.  Shared by the attention tests; uses nothing of the library."""
import math

import torch


def bucket(r, buckets, max_distance, two_sided):
    """Whole-number arithmetic: log(a/e)/log(m/e) >= i/w  <=>  a^w e^i >= m^i e^w."""
    n = buckets // 2 if two_sided else buckets
    a = abs(r) if two_sided else max(-r, 0)
    e = n // 2
    w = n - e
    at = a
    if a >= e:
        at = e + sum(a ** w * e ** i >= max_distance ** i * e ** w for i in range(1, w))
    return at + (n if two_sided and r > 0 else 0)


class Case:
    def __init__(self, batch=1, len_q=64, len_kv=None, heads_q=2, heads_kv=None, dim=64, causal=True, q_pos=None, scale=None,
                 buckets=0, max_distance=128, two_sided=False, kv_len=None):
        self.batch, self.len_q, self.len_kv = batch, len_q, len_q if len_kv is None else len_kv
        self.heads_q, self.heads_kv, self.dim = heads_q, heads_q if heads_kv is None else heads_kv, dim
        self.causal, self.q_pos = causal, self.len_kv - len_q if q_pos is None else q_pos
        self.scale = dim ** -0.5 if scale is None else scale
        self.buckets, self.max_distance, self.two_sided, self.kv_len = buckets, max_distance, two_sided, kv_len

    def inputs(self, seed=0, table_dtype=torch.float32, spread=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: (spread * torch.randn(*s, generator=g, device="cuda")).bfloat16()  # noqa: E731
        q = rnd(self.batch, self.len_q, self.heads_q, self.dim)
        k, v = (rnd(self.batch, self.len_kv, self.heads_kv, self.dim) for _ in range(2))
        dout = rnd(self.batch, self.len_q, self.heads_q, self.dim)
        table = None
        if self.buckets:
            table = (0.7 * torch.randn(self.heads_q, self.buckets, generator=g, device="cuda")).to(table_dtype)
        lens = None if self.kv_len is None else torch.tensor(self.kv_len, dtype=torch.int32, device="cuda")
        return q, k, v, dout, table, lens

    def head(self, q, k, v, table, b, h):
        """Of one head: (q, k, v in 64 bits with unused keys as zeros, scores, allowed, buckets)."""
        m = self.len_kv if self.kv_len is None else min(max(self.kv_len[b], 0), self.len_kv)
        hk = h // (self.heads_q // self.heads_kv)
        q = q[b, :, h].double()
        k, v = k[b, :, hk].double().clone(), v[b, :, hk].double().clone()
        k[m:], v[m:] = 0, 0
        i = torch.arange(self.len_q, device="cuda")[:, None] + self.q_pos
        j = torch.arange(self.len_kv, device="cuda")[None, :]
        ok = (j < m) & ((j <= i) if self.causal else (j >= 0))
        x = self.scale * (q @ k.T)
        at = None
        if self.buckets:
            lo = 1 - self.len_q - self.q_pos
            known = torch.tensor([bucket(r, self.buckets, self.max_distance, self.two_sided)
                                  for r in range(lo, self.len_kv - self.q_pos)], device="cuda")
            at = known[j - i - lo]
            t = table[h].double()
            x = x + torch.where(t <= -1e30, -math.inf, t)[at]
            ok = ok & (t > -1e30)[at]
        return q, k, v, x.masked_fill(~ok, -math.inf), ok, at

    def forward(self, q, k, v, table):
        """(o, lse, sum_j p_ij |v_j|) in 64 bits."""
        o = torch.zeros(self.batch, self.len_q, self.heads_q, self.dim, dtype=torch.float64, device="cuda")
        a = torch.zeros_like(o)
        lse = torch.full((self.batch, self.heads_q, self.len_q), -math.inf, dtype=torch.float64, device="cuda")
        if self.len_kv == 0:
            return o, lse, a
        for b in range(self.batch):
            for h in range(self.heads_q):
                _, _, vv, x, ok, _ = self.head(q, k, v, table, b, h)
                lse[b, h] = torch.logsumexp(x, 1)
                p = torch.where(ok, torch.exp(x - lse[b, h, :, None]), 0.0)
                o[b, :, h], a[b, :, h] = p @ vv, p @ vv.abs()
        return o, lse, a

    def backward(self, q, k, v, table, out, lse, dout):
        """Gradients in 64 bits from the stored out and lse, as a dict name -> (gradient, sum of |ds| |k| and its like,
        sum of p (|dp| + |delta|) |k| and its like): what the roundings of ds or p and the binary32 arithmetic scale with."""
        f64 = dict(dtype=torch.float64, device="cuda")
        shape = {"dq": q.shape, "dk": k.shape, "dv": v.shape, "dtable": (self.heads_q, max(1, self.buckets))}
        r = {n: [torch.zeros(s, **f64) for _ in range(3)] for n, s in shape.items()}
        for b in range(self.batch if self.len_kv else 0):
            for h in range(self.heads_q):
                hk = h // (self.heads_q // self.heads_kv)
                qq, kk, vv, x, ok, at = self.head(q, k, v, table, b, h)
                l = lse[b, h].double()[:, None]
                live = l != -math.inf
                do = torch.where(live, dout[b, :, h].double(), 0.0)
                o = torch.where(live, out[b, :, h].double(), 0.0)
                qq = torch.where(live, qq, 0.0)
                p = torch.where(ok & live, torch.exp(x - l), 0.0)
                dp, delta = do @ vv.T, (do * o).sum(1, keepdim=True)
                ds, wide = p * (dp - delta), p * (dp.abs() + delta.abs())
                terms = ((ds, p, 1), (ds.abs(), p, 2), (wide, p, 3))
                for n, (e, pp, i) in enumerate(terms):
                    m = (lambda t: t) if i == 1 else torch.abs
                    r["dq"][n][b, :, h] += self.scale * (e @ m(kk))
                    r["dk"][n][b, :, hk] += self.scale * (e.T @ m(qq))
                    r["dv"][n][b, :, hk] += pp.T @ m(do)
                    if at is not None:
                        r["dtable"][n][h] += torch.zeros(self.buckets, **f64).index_add_(0, at.reshape(-1), e.reshape(-1))
        return r
