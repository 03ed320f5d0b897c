"""What is not allowed takes no part, whatever its score: pairs that the causal mask or a bucket that is taken out covers, and
keys that no query sees.  Tolerances are those of the forward and backward tests.

The inputs are finite: one query and one key (or one dout and one v) share a column that is large in these two alone, so
that the one product overflows binary32 and no other does."""
import math

import pytest
import torch

import test_gpu_attn_bwd as bwd
import test_gpu_attn_fwd as fwd
from attn_ref import Case

pytestmark = pytest.mark.gpu

HUGE = 1e25                                  # bf16; its square is beyond binary32


def run(c, inputs, clean=None, dtype=torch.float32):
    """Forward and backward against the formula; `clean`: the formula's inputs, where the call's hold what must not matter."""
    q, k, v, dout, table, lens = inputs
    cq, ck, cv, cdout = clean or (q, k, v, dout)
    plan = fwd.plan_of(c, dtype)
    out, lse = fwd.outputs(c)
    plan.alsgd_attn_fwd(q, k, v, out, lse, table=table, kv_len=lens)
    fwd.compare(c, out, lse, cq, ck, cv, table)
    got = bwd.empty_grads(q, k, v, table)
    plan.alsgd_attn_bwd(q, k, v, out, lse, dout, *got[:3], table=table, dtable=got[3], kv_len=lens)
    bwd.compare(c, got, cq, ck, cv, table, out, lse, cdout)
    return out, lse, got


def overflow(q, k, v, dout, i, j, sign):
    """The score of pair (i, j), and in another column its dout . v, beyond binary32."""
    for a, b, x in ((q, k, 5), (dout, v, 3)):
        a[..., x], b[..., x] = 0.0, 0.0
        a[:, i, :, x], b[:, j, :, x] = HUGE, sign * HUGE


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("buckets", [0, 32])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("i,j", [(0, 1), (3, 60), (64, 65), (64, 127), (100, 101), (130, 250), (255, 256), (298, 299)])
def test_scores_ahead_of_the_causal_mask_may_overflow(i, j, sign, buckets, dim):
    c = Case(batch=2, len_q=300, heads_q=4, heads_kv=2, dim=dim, buckets=buckets, kv_len=(300, 270) if j < 270 else None)
    q, k, v, dout, table, lens = c.inputs()
    overflow(q, k, v, dout, i, j, sign)
    run(c, (q, k, v, dout, table, lens))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal,i,j", [(True, 30, 27), (True, 200, 197), (True, 129, 126), (True, 620, 3), (True, 699, 400),
                                        (False, 30, 27), (False, 27, 30), (False, 126, 129), (False, 620, 3), (False, 3, 620)])
def test_scores_of_buckets_that_are_taken_out_may_overflow(causal, i, j, dtype, dim):
    """A near bucket (the diagonal's tiles) and the far one of either side (tiles that have one bias)."""
    c = Case(len_q=700, heads_q=3, dim=dim, causal=causal, buckets=32, two_sided=not causal)
    q, k, v, dout, table, _ = c.inputs(table_dtype=dtype)
    per_side = 32 if causal else 16
    bucket = (3 if abs(i - j) == 3 else per_side - 1) + (16 if j > i else 0)
    table[:, bucket] = -math.inf if dtype == torch.float32 else torch.finfo(dtype).min
    overflow(q, k, v, dout, i, j, 1)
    run(c, (q, k, v, dout, table, None), dtype=dtype)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("buckets", [0, 32])
@pytest.mark.parametrize("kv_len", [None, (400, 120, 7)])
@pytest.mark.parametrize("len_q,q_pos", [(100, 50), (100, 0), (129, 200), (1, 0), (1, 7), (300, -200), (300, -299), (70, -70)])
def test_keys_that_no_query_sees_may_hold_anything(len_q, q_pos, kv_len, buckets, dim):
    """A causal call whose last query stands before the last key."""
    c = Case(batch=3, len_q=len_q, len_kv=400, heads_q=2, heads_kv=1, dim=dim, q_pos=q_pos, buckets=buckets, kv_len=kv_len)
    q, k, v, dout, table, lens = c.inputs()
    k, v = k.clone(), v.clone()
    ends = [min(m, max(0, len_q + q_pos)) for m in kv_len or (400,) * 3]
    clean = [t.clone() for t in (k, v)]
    for b, end in enumerate(ends):
        for t in clean:
            t[b, end:] = 0
        k[b, end:], v[b, end:] = math.nan, math.inf
    _, _, got = run(c, (q, k, v, dout, table, lens), (q, *clean, dout))
    for b, end in enumerate(ends):
        assert bool((got[1][b, end:] == 0).all()) and bool((got[2][b, end:] == 0).all())
