"""Refusals of the training operators: every argument is checked before anything touches a device, so these run
without one.  The pointers are never followed."""
import ctypes as C
import math

import pytest

from paper_2401_09135_b200 import binding as B

PTR = 1 << 20      # aligned, never read


def clip(descs=((PTR, 10, 0, 0),), n=None, max_norm=1.0, out=PTR, out_dtype=0, out_elems=100, stats=PTR, work=PTR,
         work_bytes=1 << 20, device=0):
    arr = (B.GradDesc * max(len(descs), 1))()
    for a, (data, numel, off, dt) in zip(arr, descs):
        a.data, a.numel, a.offset, a.dtype = data, numel, off, dt
    return B.lib().alsgd_clip_grads(arr, len(descs) if n is None else n, max_norm, out, out_dtype, out_elems, stats, work,
                                    work_bytes, device, None)


@pytest.mark.parametrize("kw", [
    dict(n=0), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(out_dtype=2), dict(stats=None),
    dict(work=None), dict(work=PTR + 128), dict(out=PTR + 2), dict(out=PTR + 1, out_dtype=1), dict(stats=PTR + 2),
    dict(descs=[(None, 10, 0, 0)]), dict(descs=[(PTR + 2, 10, 0, 0)]), dict(descs=[(PTR + 1, 10, 0, 1)]),
    dict(descs=[(PTR, 10, 0, 7)]),
])
def test_clip_refuses_bad_arguments(kw):
    assert clip(**kw) == B.E_ARG


@pytest.mark.parametrize("kw", [
    dict(device=-1), dict(device=64), dict(descs=[(PTR, 10, 91, 0)]), dict(descs=[(PTR, 101, 0, 0)]),
    dict(descs=[(PTR, 10, (1 << 64) - 5, 0)]), dict(descs=[(PTR, (1 << 64) - 1, 0, 0)]),
    dict(descs=[(PTR, 1 << 44, 0, 0)], out_elems=1 << 50),
    dict(descs=[(PTR, 1 << 42, 0, 0)] * 3, out_elems=1 << 50),
])
def test_clip_refuses_what_is_out_of_range(kw):
    assert clip(**kw) == B.E_RANGE


def test_clip_workspace():
    n = C.c_uint64()
    L = B.lib()
    assert L.alsgd_clip_grads_bytes(0, C.byref(n)) == B.E_ARG and L.alsgd_clip_grads_bytes(1, None) == B.E_ARG
    assert L.alsgd_clip_grads_bytes(1, C.byref(n)) == B.OK
    assert clip(work_bytes=n.value - 1) == B.E_NOMEM
    many = [(PTR, 10, 0, 0)] * 513
    assert clip(descs=many, work_bytes=n.value) == B.E_NOMEM


# -- attention -------------------------------------------------------------------------------------------

def attn_desc(**kw):
    d = B.AttnDesc()
    base = dict(batch=2, heads_q=4, heads_kv=2, len_q=100, len_kv=120, dim=64, flags=1, buckets=32, max_distance=128, table_dtype=0,
                q_pos=20, scale=0.125, device=0)
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


def tensor(data=PTR, b=1 << 20, s=1 << 10, h=128):
    return B.AttnTensor(data, b, s, h)


def fwd(desc=None, q=None, k=None, v=None, o=None, table=PTR, kv_len=None, lse=PTR):
    t = tensor()
    return B.lib().alsgd_attn_fwd(desc if desc is not None else attn_desc(), q or t, k or t, v or t, table, kv_len, o or t, lse, None)


def bwd(desc=None, table=PTR, dtable=PTR, kv_len=None, lse=PTR, work=PTR, work_bytes=1 << 40, **tensors):
    t = {n: tensors.get(n) or tensor() for n in ("q", "k", "v", "o", "dout", "dq", "dk", "dv")}
    return B.lib().alsgd_attn_bwd(desc if desc is not None else attn_desc(), t["q"], t["k"], t["v"], table, kv_len, t["o"], lse, t["dout"],
                                  t["dq"], t["dk"], t["dv"], dtable, work, work_bytes, None)


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("kw,status", [
    (dict(batch=0), B.E_ARG), (dict(heads_q=0), B.E_ARG), (dict(heads_kv=0), B.E_ARG), (dict(heads_kv=3), B.E_ARG),
    (dict(dim=0), B.E_ARG), (dict(dim=60), B.E_ARG), (dict(dim=136), B.E_UNSUPPORTED), (dict(flags=4), B.E_ARG),
    (dict(scale=0.0), B.E_ARG), (dict(scale=-1.0), B.E_ARG), (dict(scale=math.nan), B.E_ARG), (dict(scale=math.inf), B.E_ARG),
    (dict(buckets=257), B.E_UNSUPPORTED), (dict(buckets=1), B.E_ARG), (dict(buckets=33, flags=2), B.E_ARG), (dict(buckets=2, flags=2), B.E_ARG),
    (dict(max_distance=16), B.E_ARG), (dict(max_distance=2049), B.E_UNSUPPORTED), (dict(table_dtype=2), B.E_ARG),
    (dict(len_q=(1 << 22) + 1), B.E_RANGE), (dict(len_kv=(1 << 22) + 1), B.E_RANGE), (dict(q_pos=(1 << 22) + 1), B.E_RANGE),
    (dict(q_pos=-(1 << 22) - 1), B.E_RANGE), (dict(device=-1), B.E_RANGE), (dict(device=64), B.E_RANGE),
    (dict(batch=1 << 16, heads_q=1 << 16, heads_kv=1), B.E_RANGE),
])
def test_attention_refuses_descriptors(call, kw, status):
    assert call(desc=attn_desc(**kw)) == status


@pytest.mark.parametrize("kw", [
    dict(table=None), dict(table=PTR + 2), dict(kv_len=PTR + 2), dict(lse=None), dict(lse=PTR + 2),
    dict(q=tensor(None)), dict(q=tensor(PTR + 8)), dict(k=tensor(b=4)), dict(v=tensor(s=-8)), dict(q=tensor(h=12)),
    dict(k=tensor(s=0)), dict(k=tensor(b=1 << 39)),
])
@pytest.mark.parametrize("call", [fwd, bwd])
def test_attention_refuses_operands(call, kw):
    assert call(**kw) == B.E_ARG


@pytest.mark.parametrize("step", ["b", "s", "h"])
def test_attention_refuses_results_that_overlap(step):
    bad = tensor(**{step: 0})
    assert fwd(o=bad) == B.E_ARG
    for name in ("dq", "dk", "dv"):
        assert bwd(**{name: bad}) == B.E_ARG


def test_attention_wants_a_table_exactly_with_buckets():
    none = attn_desc(buckets=0)
    assert fwd(desc=none) == B.E_ARG and bwd(desc=none) == B.E_ARG and bwd(desc=none, table=None) == B.E_ARG
    assert bwd(dtable=None) == B.E_ARG and bwd(dtable=PTR + 2) == B.E_ARG


def test_attention_workspace():
    n = C.c_uint64()
    L = B.lib()
    assert L.alsgd_attn_bwd_bytes(None, C.byref(n)) == B.E_ARG and L.alsgd_attn_bwd_bytes(attn_desc(), None) == B.E_ARG
    assert L.alsgd_attn_bwd_bytes(attn_desc(), C.byref(n)) == B.OK and n.value > 0
    assert bwd(work_bytes=n.value - 1) == B.E_NOMEM and bwd(work=None) == B.E_ARG and bwd(work=PTR + 128) == B.E_ARG
    assert L.alsgd_attn_status(0, None) == B.E_ARG and L.alsgd_attn_status(64, C.byref(C.c_uint32())) == B.E_RANGE


@pytest.mark.parametrize("two_sided", [False, True])
def test_buckets_by_whole_numbers(two_sided):
    """Every bucket edge against log(a/e)/log(m/e) >= i/w  <=>  a^w e^i >= m^i e^w in whole numbers."""
    out = C.c_uint32()
    for buckets in (2, 4, 6, 10, 16, 32, 64, 128, 256) + (() if two_sided else (3, 5, 7, 33)):
        n = buckets // 2 if two_sided else buckets
        e = n // 2
        for m in (5, 20, 64, 100, 128, 300, 1024, 2048):
            if e < 1 or m <= e:
                continue
            d = attn_desc(buckets=buckets, max_distance=m, flags=2 if two_sided else 0)
            edges, a = [], e
            for i in range(1, n - e):
                while a ** (n - e) * e ** i < m ** i * e ** (n - e):
                    a += 1
                edges.append(a)
            for r in sorted({s * (x + k) for x in edges + [e, m] for k in (-1, 0, 1) for s in (-1, 1)} | set(range(-9, 10)) | {-(1 << 22), 1 << 22}):
                a = abs(r) if two_sided else max(-r, 0)
                want = (a if a < e else e + sum(a >= x for x in edges)) + (n if two_sided and r > 0 else 0)
                assert B.lib().alsgd_attn_bucket(d, r, C.byref(out)) == B.OK and out.value == want, (buckets, m, r)
