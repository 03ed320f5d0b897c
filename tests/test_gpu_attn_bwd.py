"""alsgd_attn_bwd against the formulas in 64 bits, taken at the forward pass's stored out and lse, and against
differences of the forward formula.

Tolerances.  ds (or p) is rounded to bf16, relative 2^-8, before the product with k, q or dout, and the gradient once
more: 2^-8 (sum |ds| |k| + |ref|), with 2 % on top; p carries the scores' binary32 error, at most 3e-5 < 2^-15 as in the
forward test, on terms p (|dp| + |delta|).  dtable sums unrounded ds: only the last part, and 2^-8 |ref| if it is bf16.
"""
import math

import pytest
import torch

from attn_ref import Case
from paper_2401_09135_b200 import binding as B
from test_gpu_attn_fwd import outputs, plan_of

pytestmark = pytest.mark.gpu

NAMES = ("dq", "dk", "dv", "dtable")


def empty_grads(q, k, v, table):
    g = [torch.full_like(t, math.nan) for t in (q, k, v)]
    return g + [None if table is None else torch.full_like(table, math.nan)]


def compare(c, got, q, k, v, table, out, lse, dout):
    assert B.alsgd_attn_status() == 0
    ref = c.backward(q, k, v, table, out, lse, dout)
    for name, g in zip(NAMES, got):
        if g is None:
            continue
        r, by_rounding, by_arithmetic = ref[name]
        tol = 2.0 ** -15 * by_arithmetic
        if name != "dtable":
            tol = tol + 1.02 * 2.0 ** -8 * (by_rounding + r.abs())
        elif g.dtype == torch.bfloat16:
            tol = tol + 1.02 * 2.0 ** -8 * r.abs()
        else:
            tol = tol + 2.0 ** -23 * r.abs()
        off = (g.double() - r).abs()
        assert bool((off <= tol).all()), (name, float((off - tol).max()), float(off.max()))


def check(c, table_dtype=torch.float32, seed=0, poison=None):
    q, k, v, dout, table, lens = c.inputs(seed, table_dtype)
    if poison:
        poison(q, k, v, dout, table)
    plan = plan_of(c, table_dtype)
    out, lse = outputs(c)
    plan.alsgd_attn_fwd(q, k, v, out, lse, table=table, kv_len=lens)
    got, again = empty_grads(q, k, v, table), empty_grads(q, k, v, table)
    plan.alsgd_attn_bwd(q, k, v, out, lse, dout, *got[:3], table=table, dtable=got[3], kv_len=lens)
    compare(c, got, q, k, v, table, out, lse, dout)
    plan.alsgd_attn_bwd(q, k, v, out, lse, dout, *again[:3], table=table, dtable=again[3], kv_len=lens)
    for x, y in zip(got, again):
        assert x is None or torch.equal(x, y), "a second call gave other bits"
    return got


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [1, 2, 31, 63, 64, 65, 127, 128, 129, 255, 256, 257, 640, 1000])
def test_lengths(n, causal, dim):
    check(Case(batch=2, len_q=n, dim=dim, causal=causal))


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 56, 72, 80, 96, 104, 120])
def test_head_sizes(dim):
    check(Case(batch=2, len_q=190, dim=dim, buckets=16))


@pytest.mark.parametrize("lens", [(1, 1), (1, 129), (1, 1000), (5, 300), (129, 500), (300, 5), (300, 129), (1000, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_unequal_lengths(lens, causal):
    check(Case(batch=2, len_q=lens[0], len_kv=lens[1], causal=causal, buckets=32, two_sided=not causal))


@pytest.mark.parametrize("q_pos", [-400, -130, -1, 0, 7, 200, 5000])
@pytest.mark.parametrize("causal", [False, True])
def test_query_positions(q_pos, causal):
    check(Case(len_q=257, len_kv=300, q_pos=q_pos, causal=causal, buckets=32, two_sided=not causal))


@pytest.mark.parametrize("heads", [(1, 1), (4, 1), (6, 2), (12, 12), (16, 4)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_shared_heads(heads, dim, causal):
    check(Case(batch=2, len_q=140, heads_q=heads[0], heads_kv=heads[1], dim=dim, causal=causal, buckets=32))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
def test_more_items_than_blocks(causal, dim):
    """Every block walks several items, empty sequences and short ones between full ones."""
    lens = [(0, 300, 1, 129, 260)[i % 5] for i in range(50)]
    check(Case(batch=50, len_q=300, heads_q=4, heads_kv=2, dim=dim, causal=causal, buckets=16, kv_len=lens))
    check(Case(batch=50, len_q=270, heads_q=4, heads_kv=4, dim=dim, causal=causal))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("batch", [1, 2, 127, 128, 129, 200])
def test_ragged_batches_of_many_sequences(batch, causal):
    """Up to 128 sequences are walked in the order of their lengths, more as they come; equal lengths and empty ones among them."""
    lens = [(97 * i + 13) % 430 if i % 7 else (0, 384, 385, 512)[i // 7 % 4] for i in range(batch)]
    check(Case(batch=batch, len_q=200, len_kv=400, heads_q=2, heads_kv=1, q_pos=150, causal=causal, buckets=16, two_sided=not causal, kv_len=lens))


@pytest.mark.parametrize("two_sided", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("buckets,max_distance", [(2, 2), (4, 5), (16, 64), (32, 128), (32, 1000), (64, 128), (256, 2048), (6, 20)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_buckets(buckets, max_distance, two_sided, causal, dtype):
    if two_sided and buckets == 2:
        pytest.skip("two sides of one bucket are refused")
    check(Case(batch=2, len_q=700, causal=causal, buckets=buckets, max_distance=max_distance, two_sided=two_sided), dtype)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("kv_len", [(0, 300, 1), (127, 128, 129), (255, 17, 256), (-5, 4000, 299)])
def test_ragged_batches_with_poison_behind_the_end(kv_len, causal, dim):
    def poison(q, k, v, dout, table):
        for b, m in enumerate(kv_len):
            m = min(max(m, 0), 300)
            k[b, m:], v[b, m:] = math.nan, math.inf
    got = check(Case(batch=3, len_q=300, dim=dim, causal=causal, buckets=32, two_sided=not causal, kv_len=kv_len), poison=poison)
    for b, m in enumerate(kv_len):
        m = min(max(m, 0), 300)
        assert bool((got[1][b, m:] == 0).all()) and bool((got[2][b, m:] == 0).all())


@pytest.mark.parametrize("q_pos", [0, 3, 40, 63, 65, 100])
def test_poison_behind_the_end_that_the_causal_mask_covers(q_pos):
    """Rows that stop before the sequence's end, in a tile that reaches behind it."""
    def poison(q, k, v, dout, table):
        for b, m in enumerate((228, 130)):
            k[b, m:], v[b, m:] = math.nan, math.inf
    check(Case(batch=2, len_q=128, len_kv=400, q_pos=q_pos, buckets=32, kv_len=(228, 130)), poison=poison)


@pytest.mark.parametrize("dim", [64, 128])
def test_rows_without_keys_take_no_part(dim):
    """More queries than keys: the first rows are empty, and whatever their q and dout hold reaches nothing."""
    def poison(q, k, v, dout, table):
        q[:, :130], dout[:, :130] = math.nan, math.inf
    got = check(Case(batch=2, len_q=300, len_kv=170, dim=dim, buckets=32), poison=poison)
    assert bool((got[0][:, :130] == 0).all())


def test_no_keys_and_no_queries():
    c = Case(batch=2, len_q=200, len_kv=0, causal=False, buckets=16, two_sided=True)
    got = check(c)
    assert bool((got[0] == 0).all()) and bool((got[3] == 0).all())
    c = Case(batch=2, len_q=0, len_kv=70, causal=False, buckets=16, two_sided=True)
    got = check(c)
    assert all(bool((g == 0).all()) for g in got[1:])


def test_buckets_that_are_taken_out():
    for lowest, dtype in ((-math.inf, torch.float32), (torch.finfo(torch.bfloat16).min, torch.bfloat16)):
        def poison(q, k, v, dout, table):
            table[0, 0] = lowest             # a token may not see itself: row 0 is empty
            table[1, 1:] = lowest            # only itself
            table[2, :15] = lowest           # only far tokens: the first rows are empty
        got = check(Case(len_q=400, heads_q=3, buckets=16, max_distance=64), dtype, poison=poison)
        assert float(got[3][0, 0]) == 0.0 and bool((got[3][1, 1:] == 0).all()) and bool((got[3][2, :15] == 0).all())


def test_strides():
    c = Case(batch=2, len_q=150, heads_q=4, heads_kv=4, buckets=32)
    q, k, v, dout, table, _ = c.inputs()
    plan = plan_of(c)
    out, lse = outputs(c)
    plan.alsgd_attn_fwd(q, k, v, out, lse, table=table)
    want = empty_grads(q, k, v, table)
    plan.alsgd_attn_bwd(q, k, v, out, lse, dout, *want[:3], table=table, dtable=want[3])
    packed, dpacked = torch.stack([q, k, v], 2), torch.full((2, 150, 3, 4, 64), math.nan, dtype=torch.bfloat16, device="cuda")
    by_head = lambda t: t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)  # noqa: E731
    dtable = torch.empty_like(table)
    plan.alsgd_attn_bwd(packed[:, :, 0], packed[:, :, 1], packed[:, :, 2], by_head(out), lse, by_head(dout), dpacked[:, :, 0],
                        dpacked[:, :, 1], dpacked[:, :, 2], table=table, dtable=dtable)
    for i in range(3):
        assert torch.equal(dpacked[:, :, i], want[i])
    assert torch.equal(dtable, want[3])
    kb, vb, db = k[:1, :, :1].expand(2, 150, 4, 64), v[:1, :, :1].expand(2, 150, 4, 64), dout[:1].expand(2, 150, 4, 64)
    plan.alsgd_attn_fwd(q, kb, vb, out, lse, table=table)
    plan.alsgd_attn_bwd(q, kb, vb, out, lse, db, *want[:3], table=table, dtable=want[3])
    compare(c, want, q, kb, vb, table, out, lse, db)


def test_another_stream_and_graph():
    c = Case(batch=2, len_q=333, buckets=32)
    q, k, v, dout, table, _ = c.inputs()
    plan = plan_of(c)
    out, lse = outputs(c)
    got = empty_grads(q, k, v, table)
    plan.alsgd_attn_fwd(q, k, v, out, lse, table=table)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    plan.alsgd_attn_bwd(q, k, v, out, lse, dout, *got[:3], table=table, dtable=got[3], stream=s)
    s.synchronize()
    compare(c, got, q, k, v, table, out, lse, dout)
    want = [g.clone() for g in got]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.alsgd_attn_fwd(q, k, v, out, lse, table=table)
        plan.alsgd_attn_bwd(q, k, v, out, lse, dout, *got[:3], table=table, dtable=got[3])
    for g in got:
        g.zero_()
    graph.replay()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_differences():
    """The loss sum(o * dout) in 64 bits, moved along each gradient: a central difference against |gradient|.  The
    gradient's roundings are below 2^-7 of it, and those of the stored out and lse of the same order: 1.5 %."""
    c = Case(batch=2, len_q=90, len_kv=110, heads_q=4, heads_kv=2, buckets=16, max_distance=64, kv_len=(110, 57))
    q, k, v, dout, table, lens = c.inputs(seed=5)
    plan = plan_of(c)
    out, lse = outputs(c)
    plan.alsgd_attn_fwd(q, k, v, out, lse, table=table, kv_len=lens)
    got = empty_grads(q, k, v, table)
    plan.alsgd_attn_bwd(q, k, v, out, lse, dout, *got[:3], table=table, dtable=got[3], kv_len=lens)
    at = [t.double() for t in (q, k, v, table)]
    for i, g in enumerate(got):
        size = float(g.double().norm())
        step = 1e-4 * g.double() / size

        def loss(sign):
            moved = [t + sign * step if n == i else t for n, t in enumerate(at)]
            return float((c.forward(*moved)[0] * dout.double()).sum())
        slope = (loss(1) - loss(-1)) / 2e-4
        assert abs(slope - size) <= 0.015 * size, (NAMES[i], slope, size)
