"""What is measured of the worker-side training operators: gradient clipping into the flat vector, attention with a
learned relative position bias, and attention's backward pass.

Every case is a dict of plain values.  `prepare` makes what a training program has in hand before the call, `run` is
one call, `work` is what the call cannot do without and `exact` its definition in 64 bits.
"""
import math

import torch

own = False

# The layouts are this repository's: the ragged test layout, its 23M / 110M parameter decoders and the paper's 150M one.
LAYOUTS = {
    "ragged": [1037, 5, 3, 4099, 1, 257, 130, 7001],
    "23m": ("decoder", 32000, 384, 384, 1536, 6),
    "110m": ("decoder", 32000, 768, 768, 3072, 12),
    "paper150m": ("decoder", 32000, 896, 1024, 3584, 12),
}
ALIGN = 128


def listed():
    return [
        # The smallest gradient list: eight tensors of odd sizes, where launches are all there is.
        dict(name="clip_ragged", op="clip", layout="ragged", layers=0, grads="f32", out="f32", clipped=True),
        # One inner step of the 23M-parameter workers with fp32 gradients; fits the L2 cache.
        dict(name="clip_23m_f32", op="clip", layout="23m", layers=6, grads="f32", out="f32", clipped=True),
        # The 110M-parameter workers after a mixed-precision backward pass: matrices in bf16, gains and biases in fp32.
        dict(name="clip_110m_mixed", op="clip", layout="110m", layers=12, grads="mixed", out="bf16", clipped=True),
        # The paper's 150M model, fp32 gradients: three times the L2 cache and more.
        dict(name="clip_150m_f32", op="clip", layout="paper150m", layers=12, grads="f32", out="f32", clipped=True),
        # A short odd prompt of one sequence: latency.
        dict(name="fwd_odd_77", op="fwd", batch=1, hq=6, hkv=6, sq=77, sk=77, dim=64, causal=True, ragged=False,
             buckets=32, max_distance=128, bidirectional=False, table="bf16"),
        # The paper's training shape: sequences of 256 tokens, 16 heads of size 64.
        dict(name="fwd_train_256", op="fwd", batch=64, hq=16, hkv=16, sq=256, sk=256, dim=64, causal=True, ragged=False,
             buckets=32, max_distance=128, bidirectional=False, table="bf16"),
        # The same model on long documents.
        dict(name="fwd_long_4096", op="fwd", batch=2, hq=16, hkv=16, sq=4096, sk=4096, dim=64, causal=True, ragged=False,
             buckets=32, max_distance=128, bidirectional=False, table="f32"),
        # Wide heads shared by groups of four, ragged batch, both directions, more keys than queries.
        dict(name="fwd_ragged_gqa", op="fwd", batch=4, hq=16, hkv=4, sq=1000, sk=1531, dim=128, causal=False, ragged=True,
             buckets=32, max_distance=256, bidirectional=True, table="f32"),
        # The backward passes of the four.
        dict(name="bwd_odd_77", op="bwd", batch=1, hq=6, hkv=6, sq=77, sk=77, dim=64, causal=True, ragged=False,
             buckets=32, max_distance=128, bidirectional=False, table="bf16"),
        dict(name="bwd_train_256", op="bwd", batch=64, hq=16, hkv=16, sq=256, sk=256, dim=64, causal=True, ragged=False,
             buckets=32, max_distance=128, bidirectional=False, table="bf16"),
        dict(name="bwd_long_4096", op="bwd", batch=2, hq=16, hkv=16, sq=4096, sk=4096, dim=64, causal=True, ragged=False,
             buckets=32, max_distance=128, bidirectional=False, table="f32"),
        dict(name="bwd_ragged_gqa", op="bwd", batch=4, hq=16, hkv=4, sq=1000, sk=1531, dim=128, causal=False, ragged=True,
             buckets=32, max_distance=256, bidirectional=True, table="f32"),
    ]


def draw(rng):
    """One more case: a layout with another number of layers, or an attention shape whose sizes spread over the range."""
    op = rng.choice(["clip", "fwd", "bwd"])
    if op == "clip":
        layout = rng.choice(["23m", "110m", "paper150m"])
        return dict(op="clip", layout=layout, layers=rng.randint(1, 12), grads=rng.choice(["f32", "bf16", "mixed"]),
                    out=rng.choice(["f32", "bf16"]), clipped=rng.random() < 0.8)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    hkv = rng.choice([1, 2, 3, 4, 6, 8])
    hq = hkv * rng.choice([1, 1, 2, 4])
    dim = rng.choice([64, 64, 64, 32, 80, 96, 128])
    causal = rng.random() < 0.7
    most = 16 * 4096 * 4096 * 64                          # the longest listed case, where half of the pairs are masked
    sq = min(log(17, 4096), math.isqrt(most // (hq * dim)) * 2 // 3)
    sk = sq + rng.choice([0, 0, 0, log(1, max(2, sq // 2))])
    return dict(op=op, batch=max(1, min(log(1, 64), most // (hq * sq * sk * dim))), hq=hq, hkv=hkv, sq=sq, sk=sk,
                dim=dim, causal=causal, ragged=rng.random() < 0.3,
                buckets=rng.choice([0, 16, 32, 32, 64]), max_distance=rng.choice([64, 128, 128, 300]),
                bidirectional=not causal, table=rng.choice(["f32", "bf16"]))


# ---------------------------------------------------------------------------------------------- inputs

def numels(case):
    spec = LAYOUTS[case["layout"]]
    if isinstance(spec, list):
        return spec
    _, vocab, width, attn, ff, _ = spec
    layer = [width, width, width * attn, width * attn, width * attn, attn * width, width, width, width * ff, ff * width]
    return [vocab * width] + layer * case["layers"] + [width, width]


def offsets(sizes):
    out, at = [], 0
    for n in sizes:
        out.append(at)
        at += -(-n // ALIGN) * ALIGN
    return out, at


def dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def kv_lengths(case):
    """Valid keys of each sequence of the batch: full without `ragged`, else spread down to a third."""
    b, sk = case["batch"], case["sk"]
    return [sk - (2 * sk * i) // (3 * b) if case["ragged"] else sk for i in range(b)]


def q_pos(case):
    return case["sk"] - case["sq"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if case["op"] == "clip":
        sizes = numels(case)
        offs, total = offsets(sizes)
        kinds = [{"f32": "f32", "bf16": "bf16"}.get(case["grads"], "bf16" if n > 8192 else "f32") for n in sizes]
        # autograd leaves each gradient in an allocation of its own; magnitudes differ from tensor to tensor
        grads = [(torch.randn(n, generator=g, device="cuda") * (1e-3 * (1 + i % 7))).to(dtype(k))
                 for i, (n, k) in enumerate(zip(sizes, kinds))]
        pads = [torch.zeros(-n % ALIGN, device="cuda") for n in sizes]
        s = dict(case=case, grads=grads, pads=pads, max_norm=0.25 if case["clipped"] else 1e4,
                 out=torch.zeros(total, dtype=dtype(case["out"]), device="cuda"), stats=torch.zeros(2, device="cuda"))
        if own:
            from paper_2401_09135_b200 import binding
            s["plan"] = binding.GradClip(sizes, offs, [dtype(k) for k in kinds], dtype(case["out"]))
        return s
    b, hq, hkv, sq, sk, d = (case[k] for k in ("batch", "hq", "hkv", "sq", "sk", "dim"))
    rnd = lambda *shape: torch.randn(*shape, generator=g, device="cuda").bfloat16()  # noqa: E731
    s = dict(case=case, q=rnd(b, sq, hq, d), k=rnd(b, sk, hkv, d), v=rnd(b, sk, hkv, d), table=None, kv_len=None)
    if case["buckets"]:
        s["table"] = (0.5 * torch.randn(hq, case["buckets"], generator=g, device="cuda")).to(dtype(case["table"]))
    if case["ragged"]:
        s["kv_len"] = torch.tensor(kv_lengths(case), dtype=torch.int32, device="cuda")
    s["out"] = torch.empty(b, sq, hq, d, dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.empty(b, hq, sq, device="cuda")
    if case["op"] == "bwd":
        # the forward pass has left its result and the rows' log-sum-exp; the layers above have left d(out)
        s["out"], s["lse"] = plain_fwd(s)
        s["dout"] = rnd(b, sq, hq, d)
        s["grads"] = [torch.empty_like(s[x]) for x in ("q", "k", "v")]
        s["dtable"] = None if s["table"] is None else torch.empty_like(s["table"])
    if own:
        from paper_2401_09135_b200 import binding
        s["plan"] = binding.Attention(b, sq, sk, hq, hkv, d, causal=case["causal"], q_pos=q_pos(case), buckets=case["buckets"],
                                      max_distance=case["max_distance"], bidirectional=case["bidirectional"],
                                      table_dtype=dtype(case["table"]))
    return s


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    if not own:
        return {"clip": plain_clip, "fwd": plain_fwd, "bwd": plain_bwd}[case["op"]](s)
    plan = s["plan"]
    if case["op"] == "clip":
        plan.alsgd_clip_grads(s["grads"], s["max_norm"], s["out"], s["stats"])
        return s["out"], s["stats"]
    if case["op"] == "fwd":
        plan.alsgd_attn_fwd(s["q"], s["k"], s["v"], s["out"], s["lse"], table=s["table"], kv_len=s["kv_len"])
        return s["out"], s["lse"]
    dq, dk, dv = s["grads"]
    plan.alsgd_attn_bwd(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], dq, dk, dv, table=s["table"],
                        dtable=s["dtable"], kv_len=s["kv_len"])
    return dq, dk, dv, s["dtable"]


def plain_clip(s):
    flat = torch.cat([x.float() for pair in zip(s["grads"], s["pads"]) for x in pair])
    norm = flat.square().sum().sqrt()
    scale = torch.where(norm <= s["max_norm"], torch.ones_like(norm), s["max_norm"] / norm)
    return (flat * scale).to(s["out"].dtype), torch.stack([norm, scale])


def bucket_of(r, case):
    """Bucket of every distance r = key position - query position (a whole-number tensor)."""
    n = case["buckets"] // 2 if case["bidirectional"] else case["buckets"]
    a = r.abs() if case["bidirectional"] else (-r).clamp(min=0)
    e = n // 2
    # the small term keeps a distance that is an exact power on its own side of the edge
    far = e + torch.floor(torch.log(a.clamp(min=1).double() / e) / math.log(case["max_distance"] / e) * (n - e) + 1e-9).long()
    at = torch.where(a < e, a, far.clamp(max=n - 1))
    return at + n * (r > 0) if case["bidirectional"] else at


def plain_scores(s):
    """(scores with bias and mask, masked places at -inf; the mask) as [batch, heads, queries, keys] in fp32."""
    case = s["case"]
    group = case["hq"] // case["hkv"]
    q = s["q"].float().permute(0, 2, 1, 3)
    k = s["k"].float().permute(0, 2, 3, 1).repeat_interleave(group, 1)
    x = (q @ k) * case["dim"] ** -0.5
    i = torch.arange(case["sq"], device="cuda")[:, None] + q_pos(case)
    j = torch.arange(case["sk"], device="cuda")[None, :]
    if s["table"] is not None:
        x += s["table"].float()[:, bucket_of(j - i, case)]
    ok = (j <= i if case["causal"] else j >= 0).expand(case["batch"], 1, case["sq"], case["sk"])
    if s["kv_len"] is not None:
        ok = ok & (j[None, None] < s["kv_len"][:, None, None, None])
    return x.masked_fill_(~ok, -math.inf), ok


def plain_fwd(s):
    group = s["case"]["hq"] // s["case"]["hkv"]
    x, _ = plain_scores(s)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = x.sum(-1, keepdim=True)
    v = s["v"].float().permute(0, 2, 1, 3).repeat_interleave(group, 1)
    o = (x @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.permute(0, 2, 1, 3).bfloat16(), (top + total.log()).squeeze(-1)


def plain_bwd(s):
    case = s["case"]
    b, hq, hkv, sq, sk, d = (case[k] for k in ("batch", "hq", "hkv", "sq", "sk", "dim"))
    group, scale = hq // hkv, d ** -0.5
    x, ok = plain_scores(s)
    lse = s["lse"][..., None]
    p = torch.exp(x - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse))
    del x
    heads = lambda t: t.float().permute(0, 2, 1, 3)  # noqa: E731
    do = heads(s["dout"])
    delta = (do * heads(s["out"])).sum(-1, keepdim=True)
    shared = lambda t: t.unflatten(1, (hkv, group)).sum(2).permute(0, 2, 1, 3).bfloat16()  # noqa: E731
    dv = shared(p.transpose(2, 3) @ do)
    ds = do @ heads(s["v"]).repeat_interleave(group, 1).transpose(2, 3)
    ds = ds.sub_(delta).mul_(p)
    del p
    dq = (ds @ heads(s["k"]).repeat_interleave(group, 1) * scale).permute(0, 2, 1, 3).bfloat16()
    dk = shared(ds.transpose(2, 3) @ heads(s["q"]) * scale)
    if s["table"] is None:
        return dq, dk, dv, None
    # row i moves right by sq - 1 - i, so that a column holds one distance; then the distances of each bucket are added
    width = sk + sq - 1
    skew = torch.nn.functional.pad(ds.sum(0).flip(1), (0, sq)).flatten(1)[:, : sq * width].view(hq, sq, width)
    by_distance = skew.sum(1)
    at = bucket_of(torch.arange(width, device="cuda") - (sq - 1) - q_pos(case), case)
    dtable = by_distance @ (at[:, None] == torch.arange(case["buckets"], device="cuda")).float()
    return dq, dk, dv, dtable.to(s["table"].dtype)


# ---------------------------------------------------------------------------------------------- what it cannot do without

def pairs(case):
    """Allowed (query, key) pairs of one head, over the batch."""
    total = 0
    for n in kv_lengths(case):
        if not case["causal"]:
            total += case["sq"] * n
            continue
        first = q_pos(case) + 1                           # keys that query 0 sees
        full = max(0, min(case["sq"], n - first + 1))     # queries before the sequence's end cuts them off
        total += full * first + full * (full - 1) // 2 + (case["sq"] - full) * n
    return total


def work(case):
    if case["op"] == "clip":
        sizes = numels(case)
        size = {"f32": 4, "bf16": 2}
        read = sum(n * (size.get(case["grads"]) or (2 if n > 8192 else 4)) for n in sizes)
        return {"bytes": read + sum(sizes) * size[case["out"]] + 8, "flops": 3 * sum(sizes)}
    b, hq, hkv, sq, sk, d = (case[k] for k in ("batch", "hq", "hkv", "sq", "sk", "dim"))
    query, keys, lse = 2 * b * sq * hq * d, 2 * hkv * d * sum(kv_lengths(case)), 4 * b * hq * sq
    table = hq * case["buckets"] * (4 if case["table"] == "f32" else 2)
    flops = 4 * hq * d * pairs(case)
    if case["op"] == "fwd":
        return {"bytes": 2 * query + 2 * keys + lse + table, "flops": flops}
    return {"bytes": 4 * query + 2 * keys + 4 * b * sk * hkv * d + lse + 2 * table, "flops": flops * 5 // 2}


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "clip":
        sizes = numels(case)
        offs, total = offsets(sizes)
        out = torch.zeros(total, dtype=torch.float64, device="cuda")
        for at, n, x in zip(offs, sizes, s["grads"]):
            out[at:at + n] = x.double()
        norm = math.sqrt(math.fsum(float((x.double() ** 2).sum()) for x in s["grads"]))
        scale = 1.0 if norm <= s["max_norm"] else s["max_norm"] / norm
        return out * scale, torch.tensor([norm, scale], dtype=torch.float64)
    b, hq, hkv, sq, sk, d = (case[k] for k in ("batch", "hq", "hkv", "sq", "sk", "dim"))
    lens, shift = kv_lengths(case), q_pos(case)
    gap = torch.arange(sk)[None, :] - torch.arange(sq)[:, None] - shift
    buckets = exact_buckets(gap, case).cuda() if case["buckets"] else None
    gap = gap.cuda()
    f64 = dict(dtype=torch.float64, device="cuda")
    o, lse = torch.zeros(b, sq, hq, d, **f64), torch.full((b, hq, sq), -math.inf, **f64)
    dq, dk, dv = torch.zeros(b, sq, hq, d, **f64), torch.zeros(b, sk, hkv, d, **f64), torch.zeros(b, sk, hkv, d, **f64)
    dt = torch.zeros(hq, max(1, case["buckets"]), **f64)
    for n in range(b):
        m = lens[n]
        allowed = (gap <= 0 if case["causal"] else torch.ones_like(gap, dtype=torch.bool))[:, :m]
        for h in range(hq):
            q, k, v = s["q"][n, :, h].double(), s["k"][n, :m, h * hkv // hq].double(), s["v"][n, :m, h * hkv // hq].double()
            e = q @ k.T / math.sqrt(d)
            if buckets is not None:
                e += s["table"][h].double()[buckets[:, :m]]
            e[~allowed] = -math.inf
            if case["op"] == "fwd":
                lse[n, h] = torch.logsumexp(e, 1)
                o[n, :, h] = torch.nan_to_num(torch.exp(e - lse[n, h, :, None])) @ v
                continue
            p = torch.nan_to_num(torch.exp(e - s["lse"][n, h].double()[:, None]))
            do = s["dout"][n, :, h].double()
            dv[n, :m, h * hkv // hq] += p.T @ do
            ds = p * (do @ v.T - (do * s["out"][n, :, h].double()).sum(1, keepdim=True))
            dq[n, :, h] = ds @ k / math.sqrt(d)
            dk[n, :m, h * hkv // hq] += ds.T @ q / math.sqrt(d)
            if buckets is not None:
                dt[h] += torch.bincount(buckets[:, :m].reshape(-1), weights=ds.reshape(-1), minlength=case["buckets"])
    if case["op"] == "fwd":
        return o, lse
    return dq, dk, dv, (dt if case["buckets"] else None)


def exact_buckets(gap, case):
    """Buckets by whole numbers alone: log(a/e)/log(m/e) >= i/w  <=>  a^w e^i >= m^i e^w."""
    n = case["buckets"] // (2 if case["bidirectional"] else 1)
    e, m = n // 2, case["max_distance"]
    w = n - e
    limits, a = [], e
    for i in range(1, w):
        while a ** w * e ** i < m ** i * e ** w:
            a += 1
        limits.append(a)
    dist = gap.abs() if case["bidirectional"] else (-gap).clamp(min=0)
    at = torch.where(dist < e, dist, e + torch.bucketize(dist, torch.tensor(limits, dtype=torch.int64), right=True))
    return at + n * (gap > 0) if case["bidirectional"] else at
