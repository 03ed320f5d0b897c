"""What is not allowed takes no part, whatever it holds.  Tolerances are those of the forward and backward tests."""
import math

import pytest
import torch

import test_gpu_attn_bwd as bwd
import test_gpu_attn_fwd as fwd
from attn_ref import Case

pytestmark = pytest.mark.gpu


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
