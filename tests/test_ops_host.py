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
