"""alsgd_attn_fwd against the formula in 64 bits.

Tolerances.  Scores are sums of exact bf16 products in binary32; the probabilities are rounded to bf16 (relative 2^-8)
before they multiply v, and o is rounded to bf16 once: |o - ref| <= 2^-8 (sum_j p_j |v_j| + |ref|), with 2 % on top for
everything done in binary32.  lse carries the binary32 error of the scores (|x| up to about 10 here, at most 16 rounded
additions of partial sums, the base-2 conversion) and of the sum: 3e-5.
"""
import math

import pytest
import torch

from attn_ref import Case
from paper_2401_09135_b200 import binding as B

pytestmark = pytest.mark.gpu


def plan_of(c, table_dtype=torch.float32):
    return B.Attention(c.batch, c.len_q, c.len_kv, c.heads_q, c.heads_kv, c.dim, causal=c.causal, scale=c.scale, q_pos=c.q_pos,
                       buckets=c.buckets, max_distance=c.max_distance, bidirectional=c.two_sided, table_dtype=table_dtype)


def outputs(c):
    return (torch.full((c.batch, c.len_q, c.heads_q, c.dim), math.nan, dtype=torch.bfloat16, device="cuda"),
            torch.full((c.batch, c.heads_q, c.len_q), math.nan, device="cuda"))


def compare(c, out, lse, q, k, v, table):
    assert B.alsgd_attn_status() == 0
    o64, lse64, a = c.forward(q, k, v, table)
    assert bool(((out.double() - o64).abs() <= 1.02 * 2.0 ** -8 * (a + o64.abs())).all()), float((out.double() - o64).abs().max())
    empty = lse64 == -math.inf
    assert bool((lse[empty] == -math.inf).all())
    assert bool((out.permute(0, 2, 1, 3)[empty] == 0).all())
    assert bool(((lse.double() - lse64)[~empty].abs() <= 3e-5).all()), float((lse.double() - lse64)[~empty].abs().max())


def check(c, table_dtype=torch.float32, seed=0):
    q, k, v, _, table, lens = c.inputs(seed, table_dtype)
    out, lse = outputs(c)
    plan = plan_of(c, table_dtype)
    plan.alsgd_attn_fwd(q, k, v, out, lse, table=table, kv_len=lens)
    compare(c, out, lse, q, k, v, table)
    again = outputs(c)
    plan.alsgd_attn_fwd(q, k, v, *again, table=table, kv_len=lens)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n", [1, 2, 31, 64, 127, 128, 129, 255, 256, 257, 640, 1000])
def test_lengths(n, causal, dim):
    check(Case(batch=2, len_q=n, dim=dim, causal=causal))


@pytest.mark.parametrize("dim", [8, 16, 24, 32, 40, 56, 72, 80, 96, 104, 120])
def test_head_sizes(dim):
    check(Case(batch=2, len_q=190, dim=dim, buckets=16))


@pytest.mark.parametrize("lens", [(1, 1), (1, 129), (1, 1000), (5, 300), (129, 500), (300, 5), (300, 129), (1000, 1)])
@pytest.mark.parametrize("causal", [False, True])
def test_unequal_lengths(lens, causal):
    """With more queries than keys and a causal mask, the first rows see nothing."""
    check(Case(batch=2, len_q=lens[0], len_kv=lens[1], causal=causal, buckets=32, two_sided=not causal))


@pytest.mark.parametrize("q_pos", [-400, -130, -1, 0, 7, 200, 5000])
def test_query_positions(q_pos):
    check(Case(len_q=257, len_kv=300, q_pos=q_pos, buckets=32))
    check(Case(len_q=257, len_kv=300, q_pos=q_pos, causal=False, buckets=32, two_sided=True))


@pytest.mark.parametrize("heads", [(1, 1), (4, 1), (6, 2), (12, 12), (16, 4)])
@pytest.mark.parametrize("dim", [64, 128])
def test_shared_heads(heads, dim):
    check(Case(batch=2, len_q=140, heads_q=heads[0], heads_kv=heads[1], dim=dim, buckets=32))


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
@pytest.mark.parametrize("buckets,max_distance", [(2, 2), (4, 5), (16, 64), (32, 128), (32, 1000), (64, 128), (256, 2048), (6, 20)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_buckets(buckets, max_distance, two_sided, dtype):
    if two_sided and buckets == 2:
        pytest.skip("two sides of one bucket are refused")
    check(Case(len_q=700, causal=not two_sided, buckets=buckets, max_distance=max_distance, two_sided=two_sided), dtype)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("kv_len", [(0, 300, 1), (127, 128, 129), (255, 17, 256), (-5, 4000, 299)])
def test_ragged_batches_with_poison_behind_the_end(kv_len, causal, dim):
    c = Case(batch=3, len_q=300, dim=dim, causal=causal, buckets=32, two_sided=not causal, kv_len=kv_len)
    q, k, v, _, table, lens = c.inputs()
    for b, m in enumerate(kv_len):
        m = min(max(m, 0), 300)
        k[b, m:], v[b, m:] = math.nan, math.inf
    out, lse = outputs(c)
    plan_of(c).alsgd_attn_fwd(q, k, v, out, lse, table=table, kv_len=lens)
    compare(c, out, lse, q, k, v, table)


@pytest.mark.parametrize("q_pos", [0, 3, 40, 63, 65, 100])
def test_poison_behind_the_end_that_the_causal_mask_covers(q_pos):
    """Rows that stop before the sequence's end, in a tile that reaches behind it."""
    c = Case(batch=2, len_q=128, len_kv=400, q_pos=q_pos, buckets=32, kv_len=(228, 130))
    q, k, v, _, table, lens = c.inputs()
    for b, m in enumerate(c.kv_len):
        k[b, m:], v[b, m:] = math.nan, math.inf
    out, lse = outputs(c)
    plan_of(c).alsgd_attn_fwd(q, k, v, out, lse, table=table, kv_len=lens)
    compare(c, out, lse, q, k, v, table)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_nonfinite_keys_reach_the_rows_that_may_see_them_only(bad):
    """A key with a NaN or an infinity (its value is finite): earlier rows of a causal mask are as without it, rows that see
    it are NaN, as the definition makes them."""
    for n, at in ((200, 70), (200, 130), (300, 299)):
        c = Case(len_q=n, heads_q=3, buckets=32)
        q, k, v, _, table, _ = c.inputs()
        k[:, at, :, 5] = bad
        out, lse = outputs(c)
        plan_of(c).alsgd_attn_fwd(q, k, v, out, lse, table=table)
        clean = k.clone()
        clean[:, at] = 0
        o64, lse64, a = c.forward(q, clean, v, table)
        assert bool(((out.double() - o64).abs() <= 1.02 * 2.0 ** -8 * (a + o64.abs()))[:, :at].all())
        assert bool(((lse.double() - lse64).abs() <= 3e-5)[:, :, :at].all())
        if math.isnan(bad):
            assert bool(out[:, at:].isnan().all()) and bool(lse[:, :, at:].isnan().all())


def test_no_keys_and_no_queries():
    check(Case(batch=2, len_q=200, len_kv=0, causal=False))
    check(Case(batch=2, len_q=0, len_kv=5, causal=False))


def test_buckets_that_are_taken_out():
    """-inf and the types' lowest values mask a bucket; rows that have no other one are empty."""
    for lowest, dtype in ((-math.inf, torch.float32), (torch.finfo(torch.float32).min, torch.float32),
                          (torch.finfo(torch.bfloat16).min, torch.bfloat16), (-math.inf, torch.bfloat16)):
        c = Case(len_q=400, heads_q=3, buckets=16, max_distance=64)
        q, k, v, _, table, _ = c.inputs(table_dtype=dtype)
        table[0, 0] = lowest             # a token may not see itself: row 0 is empty
        table[1, 1:] = lowest            # only itself
        table[2, :15] = lowest           # only far tokens: the first rows are empty
        out, lse = outputs(c)
        plan_of(c, dtype).alsgd_attn_fwd(q, k, v, out, lse, table=table)
        compare(c, out, lse, q, k, v, table)


def test_growing_scores_move_the_reference():
    """Keys whose scores rise along the row, and one that falls: the running reference is replaced many times."""
    for sign in (1, -1):
        c = Case(len_q=260, len_kv=1500, causal=False, scale=1.0, dim=64)
        q, k, v, _, _, _ = c.inputs(spread=0.05)
        q[..., 0] = 1.0
        k[..., 0] = (sign * torch.linspace(-40, 40, 1500, device="cuda")).bfloat16()[None, :, None]
        out, lse = outputs(c)
        plan_of(c).alsgd_attn_fwd(q, k, v, out, lse)
        o64, lse64, a = c.forward(q, k, v, None)
        assert bool(((out.double() - o64).abs() <= 1.02 * 2.0 ** -8 * (a + o64.abs())).all())
        assert bool(((lse.double() - lse64).abs() <= 3e-5 * 4).all())      # |x| up to 40


def test_strides():
    """Packed q/k/v of one projection, heads before positions, a broadcast over the batch and over heads."""
    c = Case(batch=2, len_q=150, heads_q=4, heads_kv=4, buckets=32)
    q, k, v, _, table, _ = c.inputs()
    packed = torch.stack([q, k, v], 2)                                   # [b, s, 3, h, d]
    out, lse = outputs(c)
    plan_of(c).alsgd_attn_fwd(packed[:, :, 0], packed[:, :, 1], packed[:, :, 2], out, lse, table=table)
    compare(c, out, lse, q, k, v, table)
    qh, kh, vh = (t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (q, k, v))
    oh = torch.full((2, 4, 150, 64), math.nan, dtype=torch.bfloat16, device="cuda").permute(0, 2, 1, 3)
    plan_of(c).alsgd_attn_fwd(qh, kh, vh, oh, lse, table=table)
    assert torch.equal(out, oh)
    kb, vb = k[:1, :, :1].expand(2, 150, 4, 64), v[:1, :, :1].expand(2, 150, 4, 64)
    plan_of(c).alsgd_attn_fwd(q, kb, vb, out, lse, table=table)
    compare(c, out, lse, q, kb, vb, table)
    wide = torch.full((2, 150, 4, 72), 7.0, dtype=torch.bfloat16, device="cuda")   # rows of 144 bytes; the rest stays
    plan_of(c).alsgd_attn_fwd(q, k, v, wide[..., :64], lse, table=table)
    compare(c, wide[..., :64], lse, q, k, v, table)
    assert bool((wide[..., 64:] == 7.0).all())


def test_another_stream_and_graph():
    c = Case(batch=2, len_q=333, buckets=32)
    q, k, v, _, table, _ = c.inputs()
    plan = plan_of(c)
    out, lse = outputs(c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    plan.alsgd_attn_fwd(q, k, v, out, lse, table=table, stream=s)
    s.synchronize()
    compare(c, out, lse, q, k, v, table)
    want = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        plan.alsgd_attn_fwd(q, k, v, out, lse, table=table)
    out.zero_()
    g.replay()
    assert torch.equal(out, want)
