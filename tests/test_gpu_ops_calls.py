"""The training operators' calls beside their arithmetic."""
import math

import pytest
import torch

from attn_ref import Case
from paper_2401_09135_b200 import binding as B
from test_gpu_attn_bwd import compare as compare_grads
from test_gpu_attn_bwd import empty_grads
from test_gpu_attn_fwd import compare, outputs, plan_of
from test_gpu_clip import NORM_TOL, inside

pytestmark = pytest.mark.gpu


def test_the_status_waits_for_every_stream():
    """A stream that does not wait for the default one is busy for some 100 ms; the answer comes behind it."""
    s = torch.cuda.Stream()
    done = torch.cuda.Event()
    assert B.alsgd_attn_status() == 0
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
        done.record()
    assert B.alsgd_attn_status() == 0
    assert done.query()


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_a_bf16_table_lies_anywhere(shift):
    """As a vector of a flat layout without alignment does."""
    c = Case(batch=2, len_q=150, buckets=32)
    q, k, v, dout, table, _ = c.inputs(table_dtype=torch.bfloat16)
    room = torch.full((3, table.numel() + shift + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    at, dat = (room[i, shift:shift + table.numel()].view(table.shape) for i in (0, 2))
    at.copy_(table)
    assert at.data_ptr() % 4 == 2 * (shift % 2)
    out, lse = outputs(c)
    plan = plan_of(c, torch.bfloat16)
    plan.alsgd_attn_fwd(q, k, v, out, lse, table=at)
    compare(c, out, lse, q, k, v, table)
    got = empty_grads(q, k, v, None)[:3]
    plan.alsgd_attn_bwd(q, k, v, out, lse, dout, *got, table=at, dtable=dat)
    compare_grads(c, got + [dat], q, k, v, table, out, lse, dout)
    assert bool((room[2, :shift] == 7.0).all()) and bool((room[2, shift + table.numel():] == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("scale", [3e37, 1.0])
@pytest.mark.parametrize("max_norm", [1.0, 1e-3, 1e30])
def test_a_norm_beyond_binary32_is_clipped_like_any(max_norm, scale, out_dtype, dtype):
    """Finite gradients whose norm is above the largest binary32 value: the norm that is reported is infinite, the factor and
    the clipped gradient are those of the norm itself.  A list of small and large values has entries that the factor
    takes below the normal range: their last place is 2^-149."""
    g = torch.Generator(device="cuda").manual_seed(0)
    grads = [(torch.randn(n, generator=g, device="cuda", dtype=torch.float64).clamp(-4, 4) * s).to(t)
             for n, t, s in ((5001, dtype, 3e37), (33, torch.float32, scale))]
    assert all(bool(torch.isfinite(x).all()) for x in grads)
    norm = math.sqrt(sum(float((x.double() ** 2).sum()) for x in grads))
    assert norm > 4e38
    plan = B.GradClip([5001, 33], [0, 5001], [dtype, torch.float32], out_dtype)
    out, stats = torch.zeros(5034, dtype=out_dtype, device="cuda"), torch.zeros(2, device="cuda")
    plan.alsgd_clip_grads(grads, max_norm, out, stats)
    assert float(stats[0]) == math.inf
    assert abs(float(stats[1]) - max_norm / norm) <= (NORM_TOL + 2.0 ** -24) * max_norm / norm + 2.0 ** -149
    ref = torch.cat([x.double() for x in grads]) * (max_norm / norm)
    normal = ref.abs() >= 2.0 ** -125
    assert inside(out[normal], ref[normal])
    last = 2.0 ** -149 if out_dtype == torch.float32 else 2.0 ** -133
    assert bool(((out.double() - ref).abs()[~normal] <= last).all())
