"""What is measured of the operators that stand before and behind a worker's attention: rotary positions, the cross entropy
over the vocabulary without its logits, and the distillation from a teacher's top logits, each forward and backward.

Every case is a dict of plain values.  `prepare` makes what a training program has in hand before the call, `run` is
one call, `work` is what the call cannot do without and `exact` its definition in 64 bits.
"""
import math

import torch

own = False


def listed():
    return [
        # A short odd prompt of one sequence: latency.
        dict(name="rope_odd_77", op="rope", inverse=False, batch=1, len=77, hq=6, hk=6, dim=64, rot=64, interleaved=False,
             base=10000.0, factor=1.0, context=0, lo=0.0, hi=0.0, amplitude=1.0, given=False, pos0=0, packed=True, dtype="bf16"),
        # The paper's training shape, sequences of 256 tokens and 16 heads of size 64: q and k lie in one packed projection.
        dict(name="rope_train_256", op="rope", inverse=False, batch=64, len=256, hq=16, hk=16, dim=64, rot=64, interleaved=False,
             base=10000.0, factor=1.0, context=0, lo=0.0, hi=0.0, amplitude=1.0, given=False, pos0=0, packed=True, dtype="bf16"),
        # The gradients of long documents: wide heads shared in groups of four, half of each head turned, scaled for a context
        # 16 times as long, positions given token by token.
        dict(name="rope_long_bwd", op="rope", inverse=True, batch=4, len=4099, hq=16, hk=4, dim=128, rot=64, interleaved=True,
             base=500000.0, factor=16.0, context=8192, lo=1.0, hi=32.0, amplitude=1.2, given=True, pos0=60000, packed=False,
             dtype="bf16"),
        # The loss of that odd prompt on the 23M-parameter model: the embedding is read once, and launches count.
        dict(name="xent_fwd_odd_77", op="xent_fwd", batch=1, len=77, vocab=32000, dim=384, ragged=False, scale=1.0, index="i64"),
        # The paper's model (hidden 896) at its training shape: every token has a label.
        dict(name="xent_fwd_train", op="xent_fwd", batch=64, len=256, vocab=32000, dim=896, ragged=False, scale=1.0, index="i64"),
        # Their backward passes.
        dict(name="xent_bwd_odd_77", op="xent_bwd", batch=1, len=77, vocab=32000, dim=384, ragged=False, scale=1.0, index="i64"),
        dict(name="xent_bwd_train", op="xent_bwd", batch=64, len=256, vocab=32000, dim=896, ragged=False, scale=1.0, index="i64"),
        # A padded batch of the 110M-parameter model: sequences end at different lengths, labels behind them are -100.
        dict(name="xent_bwd_ragged", op="xent_bwd", batch=16, len=509, vocab=32000, dim=768, ragged=True, scale=1.0, index="i64"),
        # A vocabulary of an odd size beyond the L2 cache.
        dict(name="xent_bwd_wide", op="xent_bwd", batch=8, len=1024, vocab=100003, dim=1024, ragged=False, scale=1.0, index="i32"),
        # Distillation of the 23M-parameter model, a few rows and few teacher entries.
        dict(name="distill_fwd_odd_333", op="distill_fwd", batch=1, len=333, vocab=32000, dim=384, ragged=False, scale=1.0,
             index="i64", top=17, teacher="f32"),
        # The 110M-parameter model from a teacher's 64 highest logits at temperature 2, and its backward pass on a padded batch.
        dict(name="distill_fwd_64", op="distill_fwd", batch=32, len=256, vocab=32000, dim=768, ragged=False, scale=0.5,
             index="i64", top=64, teacher="bf16"),
        dict(name="distill_bwd_64", op="distill_bwd", batch=32, len=256, vocab=32000, dim=768, ragged=True, scale=0.5,
             index="i64", top=64, teacher="bf16"),
    ]


def draw(rng):
    """One more case: sizes spread over the range between the listed ones, odd ones among them."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["rope", "rope", "xent_fwd", "xent_bwd", "distill_fwd", "distill_bwd"])
    if op == "rope":
        hk = rng.choice([1, 2, 3, 4, 6, 8, 16])
        hq = min(16, hk * rng.choice([1, 1, 2, 4]))
        dim = rng.choice([64, 64, 32, 80, 96, 128])
        n = log(1, 4 * 4099)
        scaled = rng.random() < 0.5
        return dict(op=op, inverse=rng.random() < 0.5, batch=max(1, min(log(1, 64), 4 * 4099 // n)), len=n, hq=hq, hk=hk, dim=dim,
                    rot=rng.choice([dim, dim, dim // 2, dim // 4]), interleaved=rng.random() < 0.5,
                    base=rng.choice([10000.0, 500000.0]), factor=rng.choice([2.0, 8.0, 32.0]) if scaled else 1.0,
                    context=rng.choice([2048, 8192]) if scaled else 0, lo=1.0 if scaled else 0.0,
                    hi=rng.choice([4.0, 32.0]) if scaled else 0.0, amplitude=rng.choice([1.0, 1.25]),
                    given=rng.random() < 0.5, pos0=log(1, 1 << 17) - 1, packed=rng.random() < 0.5,
                    dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    vocab, dim = log(1000, 100003), 8 * log(8, 128)
    most = 8 * 1024 * 100003 * 1024                       # the widest listed case
    rows = min(log(1, 16384), most // (vocab * dim))
    n = min(rows, log(1, 1024))
    case = dict(op=op, batch=rows // n, len=n, vocab=vocab, dim=dim, ragged=rng.random() < 0.4,
                scale=rng.choice([1.0, 1.0, 0.5, 0.3]), index=rng.choice(["i64", "i32"]))
    if op.startswith("distill"):
        case.update(top=log(1, 128), teacher=rng.choice(["f32", "bf16"]))
    return case


# ---------------------------------------------------------------------------------------------- inputs

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}


def lengths(case):
    """Tokens of each sequence that take part: all without `ragged`, else spread down to a third."""
    b, n = case["batch"], case["len"]
    return [n - (2 * n * i) // (3 * b) if case["ragged"] else n for i in range(b)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return prepare_rope(case, g) if case["op"] == "rope" else prepare_loss(case, g)


def prepare_rope(case, g):
    b, n, hq, hk, d = (case[k] for k in ("batch", "len", "hq", "hk", "dim"))
    t = DTYPES[case["dtype"]]
    if case["packed"]:
        # queries, keys and values of every token side by side, as one projection leaves them
        rows = torch.randn(b, n, hq + 2 * hk, d, generator=g, device="cuda").to(t)
        q, k = rows[:, :, :hq], rows[:, :, hq:hq + hk]
    else:
        q, k = (torch.randn(b, n, h, d, generator=g, device="cuda").to(t) for h in (hq, hk))
    s = dict(case=case, q=q, k=k, q_out=torch.empty(b, n, hq, d, dtype=t, device="cuda"),
             k_out=torch.empty(b, n, hk, d, dtype=t, device="cuda"), positions=None)
    if case["given"]:
        # documents packed into rows: each row starts somewhere else
        start = case["pos0"] + torch.randint(0, 1000, (b, 1), generator=g, device="cuda")
        s["positions"] = (start + torch.arange(n, device="cuda")).int()
    if own:
        from paper_2401_09135_b200 import binding
        s["plan"] = binding.Rotary(b, n, hq, hk, d, rot=case["rot"], interleaved=case["interleaved"], base=case["base"],
                                   factor=case["factor"], context=case["context"], turns=(case["lo"], case["hi"]),
                                   amplitude=case["amplitude"], pos0=case["pos0"], dtype=t)
    return s


def prepare_loss(case, g):
    b, n, vocab, d = (case[k] for k in ("batch", "len", "vocab", "dim"))
    rows, top = b * n, case.get("top", 0)
    w = (torch.randn(vocab, d, generator=g, device="cuda") * (2.0 / math.sqrt(d))).bfloat16()
    u = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64)
    first = (vocab ** u).long().clamp_(1, vocab) - 1      # frequent tokens have the low numbers
    # behind the last norm; a trained model points to the right token, at some positions firmly and at others less so
    x = torch.randn(rows, d, generator=g, device="cuda")
    x = (x + 5.0 * torch.rand(rows, 1, generator=g, device="cuda") * torch.nn.functional.normalize(w[first].float())).bfloat16()
    ends = torch.tensor(lengths(case), device="cuda")
    valid = (torch.arange(n, device="cuda") < ends[:, None]).reshape(rows)
    s = dict(case=case, x=x, w=w, valid=valid, loss=torch.empty(rows, device="cuda"), lse=torch.empty(rows, device="cuda"))
    if top:
        # a teacher's highest logits: the first is the token that x points to, the others lie anywhere; highest first
        gap = max(1, vocab // max(1, top))
        steps = 1 + (torch.rand(rows, top - 1, generator=g, device="cuda", dtype=torch.float64) * gap).floor().long().clamp_(max=gap - 1)
        at = torch.cat([first[:, None], first[:, None] + steps.cumsum(1)], 1) % vocab
        falls = torch.rand(rows, top, generator=g, device="cuda").cumsum(1) * (8.0 / top)
        s["teacher"] = (9.0 - falls).to(DTYPES[case["teacher"]])
        s["index"] = torch.where(valid[:, None], at, torch.full_like(at, -1)).to(DTYPES[case["index"]])
    else:
        s["index"] = torch.where(valid, first, torch.full_like(first, -100)).to(DTYPES[case["index"]])
    if case["op"].endswith("bwd"):
        # the forward pass has left the rows' log-sum-exp; the mean over the tokens that count comes back as one number
        s["lse"] = plain_logits(s)[1]
        s["dloss"] = torch.full((), 1.0 / sum(lengths(case)), device="cuda").expand(rows)
        s["dx"], s["dw"] = torch.empty_like(x), torch.empty_like(w)
    if own:
        from paper_2401_09135_b200 import binding
        s["plan"] = binding.VocabLoss(rows, vocab, d, top=top, scale=case["scale"], index_dtype=DTYPES[case["index"]],
                                      teacher_dtype=DTYPES[case["teacher"]] if top else None)
    return s


# ---------------------------------------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if not own:
        return {"rope": plain_rope, "xent_fwd": plain_fwd, "distill_fwd": plain_fwd, "xent_bwd": plain_bwd, "distill_bwd": plain_bwd}[op](s)
    plan = s["plan"]
    if op == "rope":
        plan.alsgd_rope(s["q"], s["k"], s["q_out"], s["k_out"], positions=s["positions"], inverse=s["case"]["inverse"])
        return s["q_out"], s["k_out"]
    if op == "xent_fwd":
        plan.alsgd_xent_fwd(s["x"], s["w"], s["index"], s["loss"], s["lse"])
        return s["loss"], s["lse"]
    if op == "distill_fwd":
        plan.alsgd_distill_fwd(s["x"], s["w"], s["index"], s["teacher"], s["loss"], s["lse"])
        return s["loss"], s["lse"]
    if op == "xent_bwd":
        plan.alsgd_xent_bwd(s["x"], s["w"], s["index"], s["lse"], s["dloss"], s["dx"], s["dw"])
    else:
        plan.alsgd_distill_bwd(s["x"], s["w"], s["index"], s["teacher"], s["lse"], s["dloss"], s["dx"], s["dw"])
    return s["dx"], s["dw"]


def plain_rope(s):
    case = s["case"]
    half = case["rot"] // 2
    i = torch.arange(half, dtype=torch.float64, device="cuda")
    f = torch.exp(-(2.0 * i / case["rot"]) * math.log(case["base"]))
    if case["factor"] != 1.0:
        turns = f * (case["context"] / (2.0 * math.pi))
        keep = ((turns - case["lo"]) / (case["hi"] - case["lo"])).clamp(0.0, 1.0)
        f = f * keep + f / case["factor"] * (1.0 - keep)
    pos = s["positions"]
    if pos is None:
        pos = (case["pos0"] + torch.arange(case["len"], device="cuda")).expand(case["batch"], -1)
    angle = pos[..., None].double() * f
    cos = (angle.cos() * case["amplitude"]).float()[:, :, None]
    sin = (angle.sin() * (-case["amplitude"] if case["inverse"] else case["amplitude"])).float()[:, :, None]
    out = []
    for x in (s["q"], s["k"]):
        y = x.float()
        if case["interleaved"]:
            a, c = y[..., 0:case["rot"]:2], y[..., 1:case["rot"]:2]
            turned = torch.stack([a * cos - c * sin, a * sin + c * cos], -1).flatten(-2)
        else:
            a, c = y[..., :half], y[..., half:case["rot"]]
            turned = torch.cat([a * cos - c * sin, a * sin + c * cos], -1)
        out.append(torch.cat([turned, y[..., case["rot"]:]], -1).to(x.dtype))
    return tuple(out)


def plain_logits(s):
    """(scaled logits of every row, log-sum-exp with zeros for the rows that take no part), in fp32."""
    z = (s["x"].float() @ s["w"].float().T).mul_(s["case"]["scale"])
    top = z.amax(1, keepdim=True)
    lse = (top + (z - top).exp_().sum(1, keepdim=True).log())[:, 0]
    return z, torch.where(s["valid"], lse, torch.zeros_like(lse))


def plain_teacher(s):
    """(probabilities, their logarithms) of the teacher's entries."""
    t = s["teacher"].float() * s["case"]["scale"]
    t = t - t.amax(1, keepdim=True)
    log_p = t - t.exp().sum(1, keepdim=True).log()
    return log_p.exp(), log_p


def plain_fwd(s):
    z, lse = plain_logits(s)
    at = s["index"].long().clamp(min=0)
    if "teacher" in s:
        t, log_t = plain_teacher(s)
        loss = (t * (log_t - z.gather(1, at) + lse[:, None])).sum(1)
    else:
        loss = lse - z.gather(1, at[:, None])[:, 0]
    return torch.where(s["valid"], loss, torch.zeros_like(loss)), lse


def plain_bwd(s):
    scale = s["case"]["scale"]
    x, w = s["x"].float(), s["w"].float()
    z = (x @ w.T).mul_(scale).sub_(s["lse"][:, None]).exp_()
    at = s["index"].long().clamp(min=0)
    if "teacher" in s:
        z.scatter_add_(1, at, -plain_teacher(s)[0])
    else:
        z.scatter_add_(1, at[:, None], z.new_full((len(at), 1), -1.0))
    z.mul_((torch.where(s["valid"], s["dloss"], torch.zeros_like(s["dloss"])) * scale)[:, None])
    return (z @ w).bfloat16(), (z.T @ x).bfloat16()


# ---------------------------------------------------------------------------------------------- what it cannot do without

def work(case):
    if case["op"] == "rope":
        tokens, size = case["batch"] * case["len"], 2 if case["dtype"] == "bf16" else 4
        heads = tokens * (case["hq"] + case["hk"])
        return {"bytes": 2 * heads * case["dim"] * size + (4 * tokens if case["given"] else 0), "flops": 3 * heads * case["rot"]}
    rows, used = case["batch"] * case["len"], sum(lengths(case))
    vocab, d, top = case["vocab"], case["dim"], case.get("top", 0)
    index = rows * max(1, top) * (4 if case["index"] == "i32" else 8)
    teacher = used * top * (2 if case.get("teacher") == "bf16" else 4)
    product = 2 * used * vocab * d
    if case["op"].endswith("fwd"):
        return {"bytes": 2 * d * (used + vocab) + index + teacher + 8 * rows, "flops": product}
    return {"bytes": 2 * d * (used + rows + 2 * vocab) + index + teacher + 4 * used, "flops": 3 * product}


# ---------------------------------------------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return exact_rope(case, s) if case["op"] == "rope" else exact_loss(case, s)


def exact_rope(case, s):
    """Every pair of a head as a complex number, times amplitude e^(i position frequency)."""
    rot, out = case["rot"], []
    f = []
    for i in range(rot // 2):
        v = case["base"] ** (-2 * i / rot)
        if case["factor"] != 1.0:
            part = min(1.0, max(0.0, (case["context"] * v / (2 * math.pi) - case["lo"]) / (case["hi"] - case["lo"])))
            v = (1 - part) * v / case["factor"] + part * v
        f.append(v)
    f = torch.tensor(f, dtype=torch.float64, device="cuda")
    if s["positions"] is None:
        pos = torch.arange(case["pos0"], case["pos0"] + case["len"], device="cuda").repeat(case["batch"], 1)
    else:
        pos = s["positions"]
    turn = torch.polar(torch.full_like(f, case["amplitude"]).expand(*pos.shape, -1), pos.double().unsqueeze(-1) * f).unsqueeze(2)
    if case["inverse"]:
        turn = turn.conj()
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        one, other = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        c = torch.complex(y[..., one], y[..., other]) * turn
        y[..., one], y[..., other] = c.real, c.imag
        out.append(y)
    return tuple(out)


def exact_loss(case, s):
    rows, vocab, d = case["batch"] * case["len"], case["vocab"], case["dim"]
    f64 = dict(dtype=torch.float64, device="cuda")
    w, scale = s["w"].double(), case["scale"]
    forward = case["op"].endswith("fwd")
    loss, lse = torch.zeros(rows, **f64), torch.zeros(rows, **f64)
    dx, dw = torch.zeros(rows, d, **f64), torch.zeros(vocab, d, **f64)
    used = s["valid"].nonzero()[:, 0]
    for part in used.split(2048):
        x = s["x"][part].double()
        z = scale * torch.mm(x, w.T)
        at = s["index"][part].long()
        if "teacher" in s:
            t = torch.softmax(scale * s["teacher"][part].double(), 1)
        else:
            at, t = at.unsqueeze(1), torch.ones(len(part), 1, **f64)
        if forward:
            lse[part] = torch.logsumexp(z, 1)
            loss[part] = (torch.xlogy(t, t) + t * (lse[part].unsqueeze(1) - z.gather(1, at))).sum(1)
            continue
        dz = torch.exp(z - s["lse"][part].double().unsqueeze(1)).scatter_add_(1, at, -t)
        dz *= scale * s["dloss"][part].double().unsqueeze(1)
        dx[part] = torch.mm(dz, w)
        dw += torch.mm(dz.T, x)
    return (loss, lse) if forward else (dx, dw)
