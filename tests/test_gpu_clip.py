"""alsgd_clip_grads against the formula in 64 bits.

Tolerances.  A group of at most 8 squares is summed in binary32 (relative error below 8 * 2^-24, all terms positive),
the rest in binary64; the root halves that and the result is rounded once: the norm is within 5 * 2^-24.  The factor
adds one division, the result one product: within 7 * 2^-24 before a bf16 output is rounded.  Rounding is monotone, so
a bf16 result has to lie between the rounded ends of that interval, which is one value or two neighbours.
"""
import math

import pytest
import torch

from paper_2401_09135_b200 import binding as B
from paper_2401_09135_b200 import synth

pytestmark = pytest.mark.gpu

NORM_TOL = 5 * 2.0 ** -24
OUT_TOL = 7 * 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def inside(got, ref):
    """got (fp32 or bf16) within the interval around ref (64 bits), both ends rounded to got's type."""
    low, high = ((ref.abs() * (1 + s * OUT_TOL)).float().to(got.dtype) for s in (-1, 1))
    return bool(((got.abs() >= low) & (got.abs() <= high) & (torch.signbit(got) == torch.signbit(ref))).all())


def check(grads, offsets, total, max_norm, out_dtype, want_norm=None, stream=None):
    plan = B.GradClip([g.numel() for g in grads], offsets, [g.dtype for g in grads], out_dtype)
    out = torch.full((total,), 7.0, dtype=out_dtype, device="cuda")
    stats = torch.full((2,), -1.0, device="cuda")
    plan.alsgd_clip_grads(grads, max_norm, out, stats, stream=stream)
    torch.cuda.synchronize()
    norm = want_norm if want_norm is not None else math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    factor = 1.0 if norm <= max_norm else max_norm / norm
    assert abs(float(stats[0]) - norm) <= NORM_TOL * norm
    assert abs(float(stats[1]) - factor) <= (NORM_TOL + 2 ** -24) * factor
    covered = torch.zeros(total, dtype=torch.bool, device="cuda")
    for g, off in zip(grads, offsets):
        ref = g.double() * factor
        assert inside(out[off:off + g.numel()], ref)
        covered[off:off + g.numel()] = True
    assert bool((out[~covered] == 7.0).all()), "an element outside the tensors was written"
    first, first_stats = out.clone(), stats.clone()
    plan.alsgd_clip_grads(grads, max_norm, out, stats, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(first, out) and torch.equal(first_stats, stats), "a second call gave other bits"
    return out, stats


def random_grads(sizes, dtypes, seed=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * scale).to(t) for n, t in zip(sizes, dtypes)]


@pytest.mark.parametrize("out_dtype", [F32, BF16])
@pytest.mark.parametrize("kinds", [[F32], [BF16], [F32, BF16]])
@pytest.mark.parametrize("align", [1, 4, 128])
@pytest.mark.parametrize("max_norm", [0.5, 1e9, math.inf])
def test_ragged_layout(out_dtype, kinds, align, max_norm):
    sizes = [t.numel for t in synth.ragged_tensors()]
    total, offsets = B.alsgd_layout_size(synth.ragged_tensors(), align)
    check(random_grads(sizes, [kinds[i % len(kinds)] for i in range(len(sizes))]), offsets, total, max_norm, out_dtype)


@pytest.mark.parametrize("n", [1, 2, 3, 5, 7, 8, 9, 4095, 4096, 4097, 8191, 8193, (1 << 20) + 3])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sizes(n, dtype):
    check(random_grads([n], [dtype], seed=n), [0], n, 0.25, F32)


def test_empty_tensors_and_an_empty_list_of_elements():
    g = random_grads([0, 5, 0, 9], [F32, BF16, BF16, F32])
    check(g, [0, 0, 5, 5], 14, 0.1, F32)
    out, stats = check([torch.empty(0, device="cuda")], [0], 4, 0.1, F32)
    assert stats.tolist() == [0.0, 1.0]


@pytest.mark.parametrize("shift", [1, 2, 3, 5, 7])
def test_misaligned_tensors(shift):
    base = torch.randn(20011, device="cuda")
    b16 = torch.randn(20011, device="cuda").bfloat16()
    check([base[shift:shift + 9001], b16[shift:shift + 10007]], [shift, 9100 + shift], 20000, 1.0, F32)
    check([base[shift:shift + 9001], b16[shift:shift + 10007]], [shift, 9100 + shift], 20000, 1.0, BF16)


@pytest.mark.parametrize("n", [17, 128, 129, 512, 513, 1200])
def test_many_tensors(n):
    sizes = [(i * 37) % 301 for i in range(n)]
    sizes[n // 2] = 70001
    offsets, at = [], 0
    for s in sizes:
        offsets.append(at)
        at += s
    check(random_grads(sizes, [F32 if i % 3 else BF16 for i in range(n)]), offsets, at, 0.3, F32)


def test_norm_alone():
    g = random_grads([1037, 4099], [F32, BF16])
    plan = B.GradClip([1037, 4099], [0, 0], [F32, BF16], F32)
    stats = torch.zeros(2, device="cuda")
    plan.alsgd_clip_grads(g, 0.5, None, stats)
    norm = math.sqrt(sum(float((x.double() ** 2).sum()) for x in g))
    assert abs(float(stats[0]) - norm) <= NORM_TOL * norm


def test_in_place():
    flat = torch.randn(30000, device="cuda")
    ref = flat.double().clone()
    views = [flat[:12345], flat[12345:]]
    plan = B.GradClip([12345, 30000 - 12345], [0, 12345], [F32, F32], F32)
    stats = torch.zeros(2, device="cuda")
    plan.alsgd_clip_grads(views, 1.0, flat, stats)
    ref *= 1.0 / float(ref.norm())
    assert inside(flat, ref)


@pytest.mark.parametrize("scale", [1e30, 3e37, 1e-25, 1e-38])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_extreme_magnitudes(scale, dtype):
    g = random_grads([5001, 33], [dtype, F32], scale=1.0)
    g = [(x.double() * scale).to(x.dtype) for x in g]
    norm = math.sqrt(sum(float((x.double() ** 2).sum()) for x in g))
    plan = B.GradClip([5001, 33], [0, 5001], [dtype, F32], F32)
    out, stats = torch.zeros(5034, device="cuda"), torch.zeros(2, device="cuda")
    plan.alsgd_clip_grads(g, 1.0, out, stats)
    if norm < 3.4e38:
        assert abs(float(stats[0]) - norm) <= NORM_TOL * norm + 2.0 ** -149
        if norm > 1.0:
            assert abs(float(out.double().norm()) - 1.0) < 1e-5


@pytest.mark.parametrize("where", [0, 4098, 8191, 10000])
def test_nonfinite_entries(where):
    for bad in (math.nan, math.inf, -math.inf):
        g = torch.randn(10001, device="cuda")
        g[where] = bad
        plan = B.GradClip([10001], [0], [F32], F32)
        out, stats = torch.zeros(10001, device="cuda"), torch.zeros(2, device="cuda")
        plan.alsgd_clip_grads([g], 1.0, out, stats)
        if math.isnan(bad):
            assert math.isnan(float(stats[0])) and bool(out.isnan().all())
        else:
            assert float(stats[0]) == math.inf and float(stats[1]) == 0.0
            assert bool(out[where].isnan()) and int(out.isnan().sum()) == 1 and int((out == 0).sum()) == 10000


def test_all_zero():
    out, stats = check([torch.zeros(9000, device="cuda"), -torch.zeros(77, device="cuda")], [0, 9000], 9077, 1.0, BF16)
    assert stats.tolist() == [0.0, 1.0]


def test_another_stream():
    s = torch.cuda.Stream()
    g = random_grads([123457], [F32])
    torch.cuda.synchronize()
    check(g, [0], 123457, 0.5, F32, stream=s)


def test_captured_in_a_graph():
    g = random_grads([50001, 77], [BF16, F32])
    plan = B.GradClip([50001, 77], [0, 50001], [BF16, F32], F32)
    out, stats = torch.zeros(50078, device="cuda"), torch.zeros(2, device="cuda")
    plan.alsgd_clip_grads(g, 0.5, out, stats)
    want, want_stats = out.clone(), stats.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.alsgd_clip_grads(g, 0.5, out, stats)
    out.zero_()
    graph.replay()
    graph.replay()
    assert torch.equal(out, want) and torch.equal(stats, want_stats)


def test_feeds_the_inner_step():
    """Clipped bf16 / fp32 tensors through the flat vector give the AdamW step of the clipped gradient."""
    tensors = synth.ragged_tensors()
    ctx = B.Context(tensors, 1, 1, 0.9, 0.7)
    ctx.alsgd_set_global(synth.theta0(tensors, ctx.offsets, ctx.P))
    ctx.alsgd_pull(0)
    grads = random_grads([t.numel for t in tensors], [BF16 if t.numel > 100 else F32 for t in tensors])
    flat, stats = torch.zeros(ctx.P, device="cuda"), torch.zeros(2, device="cuda")
    B.GradClip([g.numel() for g in grads], ctx.offsets, [g.dtype for g in grads], F32).alsgd_clip_grads(grads, 1.0, flat, stats)
    ctx.alsgd_inner_adamw(0, flat, 1, 1e-3)
    got = ctx.alsgd_worker_state_ptrs(0)["adam_m"].double()
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    for g, off in zip(grads, ctx.offsets):
        ref = g.double() / norm * (1 - 0.9)
        # one more product, and 1 - 0.9 rounded to 24 bits
        assert bool(((got[off:off + g.numel()] - ref).abs() <= (10 * 2.0 ** -24 + 1e-7) * ref.abs() + 1e-45).all())
    ctx.close()
