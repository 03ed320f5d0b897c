"""Rotary positions against complex numbers in 64 bits: layouts, parts of a head, scaling, positions far away, steps."""
import math

import pytest
import torch

from paper_2401_09135_b200 import binding as B
from paper_2401_09135_b200.attention import attend
from paper_2401_09135_b200.rotary import rotate

pytestmark = pytest.mark.gpu


def frequencies(rot, base, factor, context, turns):
    out = []
    for i in range(rot // 2):
        f = base ** (-2 * i / rot)
        if factor != 1:
            keep = min(1.0, max(0.0, (context * f / (2 * math.pi) - turns[0]) / (turns[1] - turns[0]))) if turns[1] else 0.0
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def reference(x, pos, f, rot, interleaved, amplitude, inverse):
    """(result, bound on its error before the last rounding)."""
    one, other = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    turn = torch.polar(torch.full_like(f, amplitude).expand(*pos.shape, -1), (pos.double()[..., None] * f) * (-1 if inverse else 1))[:, :, None]
    y = x.double().clone()
    c = torch.complex(y[..., one], y[..., other])
    size = abs(amplitude) * (c.real.abs() + c.imag.abs())
    off = torch.zeros_like(y)
    off[..., one] = off[..., other] = size
    c = c * turn
    y[..., one], y[..., other] = c.real, c.imag
    # sine and cosine to 2 steps of binary32 of an angle known to 2^-24 of a turn's half, times the amplitude, two products and a sum
    return y, off * (2 + 2 * math.pi + 2 + 2) * 2.0 ** -23


def check(x, y, pos, f, rot, interleaved, amplitude, inverse):
    want, off = reference(x, pos, f, rot, interleaved, amplitude, inverse)
    half = torch.finfo(x.dtype).eps / 2
    assert bool(((y.double() - want).abs() <= off * (1 + half) + want.abs() * half).all())
    assert torch.equal(y[..., rot:], x[..., rot:])


SHAPES = [(1, 1, 1, 1, 8, 8), (2, 77, 6, 6, 64, 64), (3, 5, 4, 1, 128, 64), (1, 300, 3, 2, 80, 80), (2, 33, 2, 2, 96, 48), (1, 40, 2, 1, 256, 256),
          (2, 9, 1, 3, 72, 20), (1, 700, 8, 8, 32, 2), (2, 64, 16, 4, 128, 128), (5, 3, 2, 2, 24, 24), (1, 4500, 12, 12, 64, 32)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_shapes(shape, interleaved, dtype):
    b, n, hq, hk, d, rot = shape
    g = torch.Generator(device="cuda").manual_seed(n)
    q, k = (torch.randn(b, n, h, d, generator=g, device="cuda").to(dtype) for h in (hq, hk))
    f = frequencies(rot, 10000.0, 1, 0, (0, 0))
    plan = B.Rotary(b, n, hq, hk, d, rot=rot, interleaved=interleaved, dtype=dtype, pos0=3)
    pos = (3 + torch.arange(n, device="cuda")).expand(b, n)
    for inverse in (False, True):
        qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        plan.alsgd_rope(q, k, qo, ko, inverse=inverse)
        check(q, qo, pos, f, rot, interleaved, 1.0, inverse)
        check(k, ko, pos, f, rot, interleaved, 1.0, inverse)
        # in place, the same bits
        q2, k2 = q.clone(), k.clone()
        plan.alsgd_rope(q2, k2, q2, k2, inverse=inverse)
        assert torch.equal(q2, qo) and torch.equal(k2, ko)


@pytest.mark.parametrize("positions", [torch.int32, torch.int64])
@pytest.mark.parametrize("factor,context,turns,amplitude", [(1, 0, (0, 0), 1.0), (4, 0, (0, 0), 1.0), (16, 8192, (1, 32), 1.25), (8, 2048, (1, 4), 1.0)])
def test_given_positions_near_and_far(positions, factor, context, turns, amplitude):
    b, n, h, d = 2, 50, 3, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(b, n, h, d, generator=g, device="cuda")
    pos = torch.randint(0, 1 << 20, (b, n), generator=g, device="cuda").to(positions)
    pos[0, 0], pos[0, 1], pos[1, 0], pos[1, 1] = 0, -5, (1 << 31) - 1, 7
    if positions == torch.int64:
        pos[0, 2] = 1 << 40
    f = frequencies(d, 500000.0, factor, context, turns)
    plan = B.Rotary(b, n, h, 0, d, base=500000.0, factor=factor, context=context, turns=turns, amplitude=amplitude, dtype=torch.float32)
    assert plan.alsgd_rope_frequencies() == pytest.approx(f.tolist(), rel=1e-13)
    out = torch.empty_like(x)
    plan.alsgd_rope(x, None, out, None, positions=pos)
    want, off = reference(x, pos, f, d, False, amplitude, False)
    # beyond 2^32 the angle itself is known to 2^-52 of its size
    angle_off = pos.double().abs()[..., None, None] * 2.0 ** -51 * x.abs().double().amax(-1, keepdim=True) * 2 * amplitude
    err = (out.double() - want).abs()
    assert bool((err <= off + want.abs() * 2.0 ** -24 + angle_off).all())


def test_steps_and_a_packed_projection():
    b, n, h, d = 3, 21, 4, 64
    rows = torch.randn(b, n, 3, h, d, device="cuda").bfloat16()
    keep = rows.clone()
    q, k, _ = rows.unbind(2)
    plan = B.Rotary(b, n, h, h, d, rot=32)
    want_q, want_k = torch.empty(b, n, h, d, device="cuda").bfloat16(), torch.empty(b, n, h, d, device="cuda").bfloat16()
    plan.alsgd_rope(q, k, want_q, want_k)
    assert torch.equal(rows, keep)
    plan.alsgd_rope(q.contiguous(), k.contiguous(), *(turned := [torch.empty(b, h, n, d, device="cuda").bfloat16().transpose(1, 2) for _ in range(2)]))
    assert torch.equal(turned[0], want_q) and torch.equal(turned[1], want_k)
    plan.alsgd_rope(q, k, q, k)
    assert torch.equal(rows[:, :, 0], want_q) and torch.equal(rows[:, :, 1], want_k) and torch.equal(rows[:, :, 2], keep[:, :, 2])


def test_a_broadcast_operand():
    plan = B.Rotary(4, 9, 2, 2, 64)
    q = torch.randn(1, 9, 1, 64, device="cuda").bfloat16().expand(4, 9, 2, 64)
    out = [torch.empty(4, 9, 2, 64, device="cuda").bfloat16() for _ in range(4)]
    plan.alsgd_rope(q, q, out[0], out[1])
    plan.alsgd_rope(q.contiguous(), q.contiguous(), out[2], out[3])
    assert torch.equal(out[0], out[2]) and torch.equal(out[1], out[3])


def test_nothing_to_turn():
    plan = B.Rotary(2, 0, 2, 2, 64)
    x = torch.empty(2, 0, 2, 64, device="cuda").bfloat16()
    plan.alsgd_rope(x, x, x, x)


def test_autograd_turns_back():
    b, n, h, d = 2, 40, 3, 64
    plan = B.Rotary(b, n, h, h, d, amplitude=1.5)
    q, k = (torch.randn(b, n, h, d, device="cuda").bfloat16().requires_grad_(True) for _ in range(2))
    wq, wk = (torch.randn(b, n, h, d, device="cuda").bfloat16() for _ in range(2))
    qo, ko = rotate(plan, q, k)
    dq, dk = torch.autograd.grad((qo * wq).sum() + (ko * wk).sum(), (q, k))
    want = [torch.empty_like(wq) for _ in range(2)]
    plan.alsgd_rope(wq, wk, *want, inverse=True)
    assert torch.equal(dq, want[0]) and torch.equal(dk, want[1])
    # gradients that arrive broadcast and transposed, and one result that is not used
    dq, dk = torch.autograd.grad(rotate(plan, q, k)[0].sum(), (q, k))
    plan.alsgd_rope(torch.ones_like(wq), torch.zeros_like(wk), *want, inverse=True)
    assert torch.equal(dq, want[0]) and not bool(dk.any())
    t = wq.permute(0, 2, 3, 1).contiguous()
    dq, = torch.autograd.grad((rotate(plan, q, k)[0].permute(0, 2, 3, 1) * t).sum(), q)
    plan.alsgd_rope(wq, wk, *want, inverse=True)
    assert torch.equal(dq, want[0])
    with pytest.raises(RuntimeError):
        g, = torch.autograd.grad((rotate(plan, q, k)[0].float() ** 2).sum(), q, create_graph=True)
        (g.float() ** 2).sum().backward()


def test_distances_are_all_that_attention_sees():
    """Moved by the same number of positions, queries and keys give the same scores."""
    b, n, h, d = 1, 60, 2, 64
    q, k, v = (torch.randn(b, n, h, d, device="cuda").bfloat16() for _ in range(3))
    plan = B.Attention(b, n, n, h, h, d)
    outs = []
    for pos0 in (0, 1000):
        outs.append(attend(plan, *rotate(B.Rotary(b, n, h, h, d, pos0=pos0), q, k), v))
    # q and k are each rounded to bf16 after the turn, differently at either place: scores are off by 2^-8 (|q||k|) / sqrt(d) each time
    q2 = q.double().norm(dim=-1).amax() * k.double().norm(dim=-1).amax() / math.sqrt(d) * 2.0 ** -8 * 4
    assert float((outs[0].double() - outs[1].double()).abs().max()) <= float(v.abs().max()) * (math.expm1(2 * float(q2)) + 2.0 ** -6)


def test_captured_and_replayed():
    plan = B.Rotary(2, 50, 4, 2, 64)
    q, k = torch.randn(2, 50, 4, 64, device="cuda").bfloat16(), torch.randn(2, 50, 2, 64, device="cuda").bfloat16()
    want = torch.empty_like(q), torch.empty_like(k)
    plan.alsgd_rope(q, k, *want)
    out = torch.empty_like(q), torch.empty_like(k)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan.alsgd_rope(q, k, *out)
    graph.replay()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_offsets_beyond_32_bits():
    """Positions 2^20 + 8 elements apart."""
    b, n, h, d = 1, 2200, 2, 64
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 10 GB")
    q = torch.randn(b, n, h, d, device="cuda").bfloat16()
    plan = B.Rotary(b, n, h, h, d)
    want = torch.empty_like(q), torch.empty_like(q)
    plan.alsgd_rope(q, q, *want)
    far = torch.empty(n * ((1 << 20) + 8), dtype=torch.bfloat16, device="cuda").view(1, n, -1)[:, :, :h * d].view(b, n, h, d)
    far.copy_(q)
    out = torch.empty_like(q)
    plan.alsgd_rope(q, far, out, far)
    assert torch.equal(out, want[0]) and torch.equal(far, want[1])
