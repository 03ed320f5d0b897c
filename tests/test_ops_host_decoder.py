"""Refusals of rotary positions and of the losses over the vocabulary: every argument is checked before anything touches a
device, so these run without one.  The pointers are never followed."""
import ctypes as C
import math

import pytest

from paper_2401_09135_b200 import binding as B

PTR = 1 << 20      # aligned, never read


def rope_desc(**kw):
    d = B.RopeDesc()
    base = dict(batch=2, heads_q=4, heads_k=2, len=100, dim=64, rot=64, flags=0, dtype=B.BF16, position_dtype=B.I32, device=0, pos0=0, base=1e4,
                factor=1.0, context=0.0, turns_low=0.0, turns_high=0.0, amplitude=1.0)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


def tensor(data=PTR, b=1 << 20, s=1 << 10, h=128):
    return B.AttnTensor(data, b, s, h)


def rope(desc=None, q=None, k=None, positions=None, q_out=None, k_out=None):
    t = tensor()
    return B.lib().alsgd_rope(desc if desc is not None else rope_desc(), q or t, k or t, positions, q_out or t, k_out or t, None)


@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), B.E_ARG), (dict(heads_q=0), B.E_ARG), (dict(dim=0), B.E_ARG), (dict(dim=60), B.E_ARG), (dict(rot=0), B.E_ARG),
    (dict(rot=33), B.E_ARG), (dict(rot=66), B.E_ARG), (dict(flags=4), B.E_ARG), (dict(dtype=2), B.E_ARG), (dict(position_dtype=0), B.E_ARG),
    (dict(base=1.0), B.E_ARG), (dict(base=math.nan), B.E_ARG), (dict(base=math.inf), B.E_ARG), (dict(factor=0.5), B.E_ARG),
    (dict(factor=math.inf), B.E_ARG), (dict(factor=math.nan), B.E_ARG), (dict(amplitude=0.0), B.E_ARG), (dict(amplitude=math.nan), B.E_ARG),
    (dict(context=-1.0), B.E_ARG), (dict(context=math.nan), B.E_ARG), (dict(turns_low=-1.0), B.E_ARG), (dict(turns_low=2.0, turns_high=2.0), B.E_ARG),
    (dict(turns_high=math.inf), B.E_ARG), (dict(turns_high=math.nan), B.E_ARG), (dict(turns_low=math.nan), B.E_ARG),
    (dict(dim=264), B.E_UNSUPPORTED), (dict(len=(1 << 22) + 1), B.E_RANGE), (dict(heads_q=1 << 16, heads_k=1), B.E_RANGE),
    (dict(batch=1 << 10, len=1 << 21), B.E_RANGE), (dict(batch=1 << 11, len=1 << 20), B.E_RANGE), (dict(device=-1), B.E_RANGE), (dict(device=64), B.E_RANGE),
])
def test_rope_refuses_descriptors(kw, status):
    assert rope(desc=rope_desc(**kw)) == status
    assert B.lib().alsgd_rope_frequencies(rope_desc(**kw), (C.c_double * 256)()) == status


@pytest.mark.parametrize("kw", [
    dict(positions=PTR + 2), dict(q=tensor(None)), dict(q=tensor(PTR + 8)), dict(k=tensor(b=4)), dict(k=tensor(s=-8)), dict(q=tensor(h=12)),
    dict(q_out=tensor(b=0)), dict(q_out=tensor(s=0)), dict(k_out=tensor(h=0)), dict(k=tensor(b=1 << 39)),
])
def test_rope_refuses_operands(kw):
    assert rope(**kw) == B.E_ARG


def test_rope_refuses_nothing_at_all():
    L = B.lib()
    t = tensor()
    assert L.alsgd_rope(None, t, t, None, t, t, None) == B.E_ARG and L.alsgd_rope(rope_desc(), None, t, None, t, t, None) == B.E_ARG
    assert L.alsgd_rope(rope_desc(), t, None, None, t, t, None) == B.E_ARG and L.alsgd_rope_frequencies(rope_desc(), None) == B.E_ARG
    assert rope(desc=rope_desc(position_dtype=B.I64), positions=PTR + 4) == B.E_ARG
    assert rope(desc=rope_desc(dtype=B.F32), q=tensor(h=130)) == B.E_ARG
    assert rope(q=tensor(s=1 << 31)) == B.E_RANGE and rope(k_out=tensor(h=1 << 31)) == B.E_RANGE
    assert L.alsgd_rope(rope_desc(len=0), None, None, None, None, None, None) == B.OK


@pytest.mark.parametrize("kw", [dict(), dict(rot=32, base=5e5), dict(factor=4.0), dict(factor=16.0, context=8192.0, turns_low=1.0, turns_high=32.0)])
def test_frequencies(kw):
    d = rope_desc(**kw)
    out = (C.c_double * (d.rot // 2))()
    assert B.lib().alsgd_rope_frequencies(d, out) == B.OK
    for i, f in enumerate(out):
        want = d.base ** (-2 * i / d.rot)
        if d.factor != 1:
            keep = min(1.0, max(0.0, (d.context * want / (2 * math.pi) - d.turns_low) / (d.turns_high - d.turns_low))) if d.turns_high else 0.0
            want = keep * want + (1 - keep) * want / d.factor
        assert f == pytest.approx(want, rel=1e-13)


# -- losses over the vocabulary ------------------------------------------------------------------------------

def vocab_desc(**kw):
    d = B.VocabDesc()
    base = dict(rows=100, vocab=1000, dim=64, top=0, index_dtype=B.I64, teacher_dtype=B.F32, scale=1.0, device=0)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


def matrix(data=PTR, step=64):
    return B.Matrix(data, step)


def call(name, desc=None, x=None, w=None, index=PTR, teacher=PTR, loss=PTR, lse=PTR, dloss=PTR, dloss_step=1, dx=None, dw=None, work=PTR, work_bytes=1 << 50):
    top = name.startswith("distill")
    desc = desc if desc is not None else vocab_desc()
    if top and desc.top == 0:
        desc.top = 5
    m, to = matrix(step=max(64, desc.dim)), matrix(2 * PTR, max(64, desc.dim))
    labels = (index, teacher) if top else (index,)
    rest = (loss, lse) if name.endswith("fwd") else (lse, dloss, dloss_step, dx or to, dw or to)
    return getattr(B.lib(), "alsgd_" + name)(desc, x or m, w or m, *labels, *rest, work, work_bytes, None)


CALLS = ["xent_fwd", "xent_bwd", "distill_fwd", "distill_bwd"]


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("kw,status", [
    (dict(vocab=0), B.E_ARG), (dict(dim=0), B.E_ARG), (dict(dim=60), B.E_ARG), (dict(index_dtype=0), B.E_ARG), (dict(scale=0.0), B.E_ARG),
    (dict(scale=-1.0), B.E_ARG), (dict(scale=math.nan), B.E_ARG), (dict(scale=math.inf), B.E_ARG), (dict(scale=3e38), B.E_ARG),
    (dict(dim=16392), B.E_UNSUPPORTED), (dict(top=129), B.E_UNSUPPORTED), (dict(rows=(1 << 22) + 1), B.E_RANGE), (dict(vocab=(1 << 22) + 1), B.E_RANGE),
    (dict(device=-1), B.E_RANGE), (dict(device=64), B.E_RANGE),
])
def test_vocab_refuses_descriptors(name, kw, status):
    assert call(name, desc=vocab_desc(**kw)) == status


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("kw", [
    dict(index=None), dict(index=PTR + 4), dict(lse=None), dict(lse=PTR + 2), dict(x=matrix(None)), dict(x=matrix(PTR + 8)), dict(x=matrix(step=-64)),
    dict(x=matrix(step=68)), dict(w=matrix(step=0)), dict(w=matrix(step=56)), dict(w=matrix(None)), dict(w=matrix(step=1 << 39)), dict(work=None),
    dict(work=PTR + 128),
])
def test_vocab_refuses_operands(name, kw):
    assert call(name, **kw) == B.E_ARG


@pytest.mark.parametrize("name", ["xent_bwd", "distill_bwd"])
@pytest.mark.parametrize("kw", [dict(dloss=None), dict(dloss=PTR + 2), dict(dloss_step=-1), dict(dx=matrix(step=0)), dict(dx=matrix(step=56)),
                                dict(dw=matrix(step=56)), dict(dw=matrix(PTR + 8)), dict(dx=matrix(None)), dict(dx=matrix()), dict(dw=matrix())])
def test_vocab_refuses_gradients(name, kw):
    assert call(name, **kw) == B.E_ARG


def test_vocab_refuses_the_rest():
    L = B.lib()
    n = C.c_uint64()
    assert call("xent_fwd", desc=vocab_desc(top=5)) == B.E_ARG and call("xent_bwd", desc=vocab_desc(top=5)) == B.E_ARG
    assert call("distill_fwd", teacher=None) == B.E_ARG and call("distill_bwd", teacher=PTR + 2) == B.E_ARG
    assert call("distill_fwd", desc=vocab_desc(top=5, teacher_dtype=7)) == B.E_ARG
    assert call("xent_fwd", loss=None) == B.E_ARG and call("distill_fwd", loss=PTR + 1) == B.E_ARG
    m = matrix()
    assert L.alsgd_distill_fwd(vocab_desc(), m, m, PTR, PTR, PTR, PTR, PTR, 1 << 40, None) == B.E_ARG
    assert L.alsgd_xent_fwd(None, m, m, PTR, PTR, PTR, PTR, 1 << 40, None) == B.E_ARG
    assert L.alsgd_vocab_bytes(None, 0, C.byref(n)) == B.E_ARG and L.alsgd_vocab_bytes(vocab_desc(), 0, None) == B.E_ARG
    assert L.alsgd_vocab_status(0, None) == B.E_ARG and L.alsgd_vocab_status(64, C.byref(C.c_uint32())) == B.E_RANGE
    for name in CALLS:
        d = vocab_desc(top=5 if name.startswith("distill") else 0)
        assert L.alsgd_vocab_bytes(d, int(name.endswith("bwd")), C.byref(n)) == B.OK and n.value > 0
        assert call(name, desc=d, work_bytes=n.value - 1) == B.E_NOMEM
    # without rows there is nothing to do and nothing is looked at
    assert L.alsgd_xent_fwd(vocab_desc(rows=0), m, m, None, None, None, None, 0, None) == B.OK


def test_vocab_workspace_stays_near_a_piece():
    """The backward pass holds a piece of dz, not all of it, and no more of dw's sums than of either."""
    n = C.c_uint64()
    d = vocab_desc(rows=1 << 16, vocab=1 << 17, dim=1024)
    assert B.lib().alsgd_vocab_bytes(d, 1, C.byref(n)) == B.OK
    assert n.value < (512 << 20) + (1 << 16) * (1024 * 6 + 64) + (256 << 20) + (1 << 20)
