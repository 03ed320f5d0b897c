"""Thin ctypes binding of the C ABI declared in include/alsgd.h.

Argument marshalling only: every step of the server path and of the inner optimizer runs in the
library's CUDA kernels.  There is no CPU fallback; loading fails loudly when libalsgd.so is missing
and cannot be built.  PyTorch is used for the device arena, the stream and tensor views of the
borrowed device pointers.
"""
from __future__ import annotations

import ctypes as C
import operator
import os
import threading

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libalsgd.so")

OK, E_ARG, E_RANGE, E_STATE, E_CUDA, E_NOMEM, E_UNSUPPORTED, E_BOUNDS = 0, -1, -2, -3, -4, -5, -6, -7
TENSOR_DECAY = 1
PG_DISPATCH, PG_CURRENT = 0, 1
CFG_REPLICA_BF16, CFG_GRAD_STAGING, CFG_OUTER_BUFFERED, CFG_OUTER_SGDM, CFG_STABLE_PTRS = 1, 2, 4, 8, 16
STALE_NONE, STALE_POLY, STALE_POLY_THRES = 0, 1, 2
ARRIVE_RESEED, ARRIVE_NORM, ARRIVE_NANCHECK = 1, 2, 4
F32, BF16, I32, I64 = 0, 1, 2, 3
ATTN_CAUSAL, ATTN_BIAS_TWO_SIDED = 1, 2
ROPE_INTERLEAVED, ROPE_INVERSE = 1, 2


class TensorDesc(C.Structure):
    _fields_ = [("numel", C.c_uint64), ("flags", C.c_uint32), ("reserved", C.c_uint32)]


class Config(C.Structure):
    _fields_ = [("n_workers", C.c_uint32), ("N", C.c_uint32), ("pg_base", C.c_uint32), ("flags", C.c_uint32),
                ("beta", C.c_float), ("outer_lr", C.c_float), ("c", C.c_float),
                ("adam_b1", C.c_float), ("adam_b2", C.c_float), ("adam_eps", C.c_float), ("adam_wd", C.c_float),
                ("device", C.c_int32), ("stream", C.c_void_p), ("arena", C.c_void_p), ("arena_bytes", C.c_uint64)]


class ArrivalInfo(C.Structure):
    _fields_ = [("tick", C.c_uint64), ("staleness", C.c_uint64), ("gnorm2", C.c_double),
                ("worker", C.c_uint32), ("boundary", C.c_uint32), ("nonfinite", C.c_uint32), ("dropped", C.c_uint32)]


class ArriveOpts(C.Structure):
    _fields_ = [("weights", C.POINTER(C.c_float)), ("dc_lambda", C.c_float), ("staleness_rule", C.c_uint32),
                ("stale_threshold", C.c_uint32), ("reserved", C.c_uint32)]


class Ptrs(C.Structure):
    _fields_ = [("theta", C.c_void_p), ("m", C.c_void_p), ("delta", C.c_void_p), ("P", C.c_uint64),
                ("n_workers", C.c_uint32), ("reserved", C.c_uint32)]


class WorkerPtrs(C.Structure):
    _fields_ = [("p", C.c_void_p), ("base", C.c_void_p), ("adam_m", C.c_void_p), ("adam_v", C.c_void_p),
                ("replica", C.c_void_p)]


class LrSched(C.Structure):
    _fields_ = [("eta_max", C.c_double), ("eta_min", C.c_double), ("t_warmup", C.c_uint64), ("T", C.c_uint64)]


class GradDesc(C.Structure):
    _fields_ = [("data", C.c_void_p), ("numel", C.c_uint64), ("offset", C.c_uint64), ("dtype", C.c_uint32),
                ("reserved", C.c_uint32)]


class AttnDesc(C.Structure):
    _fields_ = [("batch", C.c_uint32), ("heads_q", C.c_uint32), ("heads_kv", C.c_uint32), ("len_q", C.c_uint32),
                ("len_kv", C.c_uint32), ("dim", C.c_uint32), ("flags", C.c_uint32), ("buckets", C.c_uint32),
                ("max_distance", C.c_uint32), ("table_dtype", C.c_uint32), ("q_pos", C.c_int32), ("scale", C.c_float),
                ("device", C.c_int32), ("reserved", C.c_uint32)]


class AttnTensor(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_batch", C.c_int64), ("stride_pos", C.c_int64), ("stride_head", C.c_int64)]


class RopeDesc(C.Structure):
    _fields_ = [("batch", C.c_uint32), ("heads_q", C.c_uint32), ("heads_k", C.c_uint32), ("len", C.c_uint32), ("dim", C.c_uint32),
                ("rot", C.c_uint32), ("flags", C.c_uint32), ("dtype", C.c_uint32), ("position_dtype", C.c_uint32), ("device", C.c_int32),
                ("pos0", C.c_int64), ("base", C.c_double), ("factor", C.c_double), ("context", C.c_double), ("turns_low", C.c_double),
                ("turns_high", C.c_double), ("amplitude", C.c_double)]


class VocabDesc(C.Structure):
    _fields_ = [("rows", C.c_uint32), ("vocab", C.c_uint32), ("dim", C.c_uint32), ("top", C.c_uint32), ("index_dtype", C.c_uint32),
                ("teacher_dtype", C.c_uint32), ("scale", C.c_float), ("device", C.c_int32)]


class Matrix(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_row", C.c_int64)]


_vp = C.c_void_p
_u32p = C.POINTER(C.c_uint32)
_u64p = C.POINTER(C.c_uint64)
_f64p = C.POINTER(C.c_double)

# name -> (restype, argtypes): every function include/alsgd.h declares
SIGNATURES = {
    "alsgd_strerror": (C.c_char_p, [C.c_int]),
    "alsgd_layout_size": (C.c_int, [C.POINTER(TensorDesc), C.c_uint32, C.c_uint32, _u64p, _u64p]),
    "alsgd_arena_bytes": (C.c_int, [C.POINTER(TensorDesc), C.c_uint32, C.c_uint32, C.POINTER(Config), _u64p]),
    "alsgd_init": (C.c_int, [C.POINTER(_vp), C.POINTER(TensorDesc), C.c_uint32, C.c_uint32, C.POINTER(Config)]),
    "alsgd_destroy": (C.c_int, [_vp]),
    "alsgd_set_global": (C.c_int, [_vp, _vp, C.c_int]),
    "alsgd_get_global": (C.c_int, [_vp, _vp, C.c_int]),
    "alsgd_set_worker_params": (C.c_int, [_vp, C.c_uint32, _vp, C.c_int]),
    "alsgd_get_worker_params": (C.c_int, [_vp, C.c_uint32, _vp, C.c_int]),
    "alsgd_pull": (C.c_int, [_vp, C.c_uint32]),
    "alsgd_inner_adamw": (C.c_int, [_vp, C.c_uint32, _vp, C.c_int, C.c_uint64, C.c_float]),
    "alsgd_inner_adamw_bf16": (C.c_int, [_vp, C.c_uint32, _vp, C.c_int, C.c_uint64, C.c_float]),
    "alsgd_arrive": (C.c_int, [_vp, _u32p, C.c_uint32, C.c_uint32, C.POINTER(ArrivalInfo)]),
    "alsgd_arrive_ex": (C.c_int, [_vp, _u32p, C.c_uint32, C.c_uint32, C.POINTER(ArriveOpts), C.POINTER(ArrivalInfo)]),
    "alsgd_counters": (C.c_int, [_vp, _u64p, _u32p]),
    "alsgd_state_ptrs": (C.c_int, [_vp, C.POINTER(Ptrs)]),
    "alsgd_worker_state_ptrs": (C.c_int, [_vp, C.c_uint32, C.POINTER(WorkerPtrs)]),
    "alsgd_state_bytes": (C.c_int, [_vp, _u64p]),
    "alsgd_export_state": (C.c_int, [_vp, _vp, C.c_uint64]),
    "alsgd_import_state": (C.c_int, [_vp, _vp, C.c_uint64]),
    "alsgd_sync": (C.c_int, [_vp]),
    "alsgd_debug_word_ptr": (C.c_int, [_vp, C.POINTER(_vp)]),
    "alsgd_debug_guard_limit": (C.c_int, [_vp, C.c_uint64]),
    "alsgd_last_cuda_error": (C.c_int, [_vp]),
    "alsgd_dylu_steps": (C.c_int, [_f64p, C.c_uint32, C.c_uint32, _u32p]),
    "alsgd_shard_probs": (C.c_int, [_f64p, _f64p, C.c_uint32, _f64p]),
    "alsgd_lr_at": (C.c_int, [C.POINTER(LrSched), C.c_uint64, _f64p]),
    "alsgd_sched_create": (C.c_int, [C.POINTER(_vp), C.c_uint32, C.c_double, C.c_uint64]),
    "alsgd_sched_destroy": (C.c_int, [_vp]),
    "alsgd_sched_dispatch": (C.c_int, [_vp, C.c_uint32, C.c_double, C.c_uint32]),
    "alsgd_sched_next_batch": (C.c_int, [_vp, _u32p, _f64p, C.c_uint32, _u32p, _f64p]),
    "alsgd_sched_local_updates": (C.c_int, [_vp, _u64p]),
    "alsgd_sched_state_bytes": (C.c_int, [_vp, _u64p]),
    "alsgd_sched_export": (C.c_int, [_vp, _vp, C.c_uint64]),
    "alsgd_sched_import": (C.c_int, [_vp, _vp, C.c_uint64]),
    "alsgd_pg_norm_static": (C.c_int, [_vp, _vp, C.c_uint64, C.c_int32, _vp, _vp, _vp]),
    "alsgd_clip_grads_bytes": (C.c_int, [C.c_uint32, _u64p]),
    "alsgd_clip_grads": (C.c_int, [C.POINTER(GradDesc), C.c_uint32, C.c_float, _vp, C.c_uint32, C.c_uint64, _vp, _vp, C.c_uint64,
                                   C.c_int32, _vp]),
    "alsgd_attn_fwd": (C.c_int, [C.POINTER(AttnDesc)] + [C.POINTER(AttnTensor)] * 3 + [_vp, _vp, C.POINTER(AttnTensor), _vp, _vp]),
    "alsgd_attn_bwd_bytes": (C.c_int, [C.POINTER(AttnDesc), _u64p]),
    "alsgd_attn_bwd": (C.c_int, [C.POINTER(AttnDesc)] + [C.POINTER(AttnTensor)] * 3 + [_vp, _vp, C.POINTER(AttnTensor), _vp]
                       + [C.POINTER(AttnTensor)] * 4 + [_vp, _vp, C.c_uint64, _vp]),
    "alsgd_attn_bucket": (C.c_int, [C.POINTER(AttnDesc), C.c_int32, _u32p]),
    "alsgd_attn_status": (C.c_int, [C.c_int32, _u32p]),
    "alsgd_rope": (C.c_int, [C.POINTER(RopeDesc)] + [C.POINTER(AttnTensor)] * 2 + [_vp] + [C.POINTER(AttnTensor)] * 2 + [_vp]),
    "alsgd_rope_frequencies": (C.c_int, [C.POINTER(RopeDesc), _f64p]),
    "alsgd_vocab_bytes": (C.c_int, [C.POINTER(VocabDesc), C.c_int, _u64p]),
    "alsgd_xent_fwd": (C.c_int, [C.POINTER(VocabDesc)] + [C.POINTER(Matrix)] * 2 + [_vp] * 4 + [C.c_uint64, _vp]),
    "alsgd_xent_bwd": (C.c_int, [C.POINTER(VocabDesc)] + [C.POINTER(Matrix)] * 2 + [_vp] * 3 + [C.c_int64] + [C.POINTER(Matrix)] * 2
                       + [_vp, C.c_uint64, _vp]),
    "alsgd_distill_fwd": (C.c_int, [C.POINTER(VocabDesc)] + [C.POINTER(Matrix)] * 2 + [_vp] * 5 + [C.c_uint64, _vp]),
    "alsgd_distill_bwd": (C.c_int, [C.POINTER(VocabDesc)] + [C.POINTER(Matrix)] * 2 + [_vp] * 4 + [C.c_int64] + [C.POINTER(Matrix)] * 2
                          + [_vp, C.c_uint64, _vp]),
    "alsgd_vocab_status": (C.c_int, [C.c_int32, _u32p]),
}
STATIC_MAX_ELEMS = 1 << 27

_lib = None
_variant = "main"


def use_debug_library(on: bool = True):
    """Route every later call through libalsgd_dbg.so (kernels with bounds checks; alsgd_sync reports refused
    accesses) instead of libalsgd.so.  Must be chosen before the first call that loads a library."""
    global _variant
    want = "debug" if on else "main"
    if _lib is not None and want != _variant:
        raise RuntimeError("a library is already loaded in this process")
    _variant = want


class AlsgdError(RuntimeError):
    def __init__(self, status, where, cuda=0):
        self.status = status
        msg = f"{where}: status {status}"
        try:
            msg += f" ({lib().alsgd_strerror(status).decode()})"
        except Exception:
            pass
        if cuda:
            msg += f", cudaError {cuda}"
        super().__init__(msg)


def lib():
    """Load libalsgd.so (building it in-tree first if the sources are newer)."""
    global _lib
    if _lib is None:
        from . import build as _build
        if _build.needs_build(_variant):
            _build.build(targets=(_variant,))
        path = LIB_PATH if _variant == "main" else _build.LIB_DBG
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: the CUDA library is required, there is no fallback")
        L = C.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)      # AttributeError if the library does not export a declared symbol
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _check(status, where, ctx=None):
    if status != OK:
        cuda = lib().alsgd_last_cuda_error(ctx) if ctx else 0
        raise AlsgdError(status, where, cuda)


def tensor_table(tensors):
    """ctypes array from an iterable of (numel, decay) pairs or objects with .numel / .decay."""
    items = [(t.numel, t.decay) if hasattr(t, "numel") else t for t in tensors]
    arr = (TensorDesc * len(items))()
    for i, (n, d) in enumerate(items):
        arr[i].numel, arr[i].flags = int(n), TENSOR_DECAY if d else 0
    return arr


def alsgd_layout_size(tensors, align_elems=128):
    tab = tensor_table(tensors)
    P = C.c_uint64()
    offs = (C.c_uint64 * len(tab))()
    _check(lib().alsgd_layout_size(tab, len(tab), align_elems, C.byref(P), offs), "alsgd_layout_size")
    return int(P.value), [int(x) for x in offs]


def alsgd_dylu_steps(speeds, H):
    sp = (C.c_double * len(speeds))(*[float(x) for x in speeds])
    out = (C.c_uint32 * len(speeds))()
    _check(lib().alsgd_dylu_steps(sp, len(speeds), int(H), out), "alsgd_dylu_steps")
    return [int(x) for x in out]


def alsgd_shard_probs(sizes, learned):
    n = len(sizes)
    s = (C.c_double * n)(*[float(x) for x in sizes])
    l = (C.c_double * n)(*[float(x) for x in learned])
    out = (C.c_double * n)()
    _check(lib().alsgd_shard_probs(s, l, n, out), "alsgd_shard_probs")
    return [float(x) for x in out]


def alsgd_lr_at(eta_max, eta_min, t_warmup, T, t):
    s = LrSched(float(eta_max), float(eta_min), int(t_warmup), int(T))
    out = C.c_double()
    _check(lib().alsgd_lr_at(C.byref(s), int(t), C.byref(out)), "alsgd_lr_at")
    return float(out.value)


class Scheduler:
    """alsgd_sched_*: Algorithm 2 / Algorithm 5 on faked time."""

    def __init__(self, n_workers, tau_grace, t_max=0):
        self._h = _vp()
        self.n = int(n_workers)
        _check(lib().alsgd_sched_create(C.byref(self._h), self.n, float(tau_grace), int(t_max)), "alsgd_sched_create")

    def dispatch(self, worker, duration, local_updates):
        _check(lib().alsgd_sched_dispatch(self._h, int(worker), float(duration), int(local_updates)), "alsgd_sched_dispatch")

    def next_batch(self):
        ids = (C.c_uint32 * self.n)()
        times = (C.c_double * self.n)()
        k = C.c_uint32()
        restart = C.c_double()
        _check(lib().alsgd_sched_next_batch(self._h, ids, times, self.n, C.byref(k), C.byref(restart)), "alsgd_sched_next_batch")
        return [int(ids[i]) for i in range(k.value)], [float(times[i]) for i in range(k.value)], float(restart.value)

    def local_updates(self):
        out = C.c_uint64()
        _check(lib().alsgd_sched_local_updates(self._h, C.byref(out)), "alsgd_sched_local_updates")
        return int(out.value)

    def export_state(self) -> bytes:
        n = C.c_uint64()
        _check(lib().alsgd_sched_state_bytes(self._h, C.byref(n)), "alsgd_sched_state_bytes")
        buf = C.create_string_buffer(int(n.value))
        _check(lib().alsgd_sched_export(self._h, buf, int(n.value)), "alsgd_sched_export")
        return buf.raw

    def import_state(self, image: bytes):
        _check(lib().alsgd_sched_import(self._h, image, len(image)), "alsgd_sched_import")

    def close(self):
        if self._h:
            lib().alsgd_sched_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Context:
    """One alsgd_ctx with a torch-owned arena on one CUDA device.  Method names follow the ABI."""

    def __init__(self, tensors, n_workers, N, beta, outer_lr, c=0.0, pg_base=PG_DISPATCH,
                 adam=(0.9, 0.95, 1e-8, 0.1), replica=True, grad_staging=False, align_elems=128,
                 device=0, stream=None, buffered=False, sgdm=False, stable_ptrs=False):
        import torch
        self.torch = torch
        if not torch.cuda.is_available():
            raise RuntimeError("alsgd needs a CUDA device; there is no CPU path")
        self.device = torch.device("cuda", device)
        self.tab = tensor_table(tensors)
        self.align = int(align_elems)
        self.P, self.offsets = alsgd_layout_size(tensors, self.align)
        cfg = Config()
        cfg.n_workers, cfg.N, cfg.pg_base = int(n_workers), int(N), int(pg_base)
        cfg.flags = ((CFG_REPLICA_BF16 if replica else 0) | (CFG_GRAD_STAGING if grad_staging else 0)
                     | (CFG_OUTER_BUFFERED if buffered else 0) | (CFG_OUTER_SGDM if sgdm else 0)
                     | (CFG_STABLE_PTRS if stable_ptrs else 0))
        cfg.beta, cfg.outer_lr, cfg.c = float(beta), float(outer_lr), float(c)
        cfg.adam_b1, cfg.adam_b2, cfg.adam_eps, cfg.adam_wd = [float(x) for x in adam]
        cfg.device = device
        nbytes = C.c_uint64()
        _check(lib().alsgd_arena_bytes(self.tab, len(self.tab), self.align, C.byref(cfg), C.byref(nbytes)), "alsgd_arena_bytes")
        self.arena_bytes = int(nbytes.value)
        with torch.cuda.device(self.device):
            self.arena = torch.empty(self.arena_bytes + 256, dtype=torch.uint8, device=self.device)
            self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        pad = (-self.arena.data_ptr()) % 256
        cfg.arena, cfg.arena_bytes = self.arena.data_ptr() + pad, self.arena_bytes
        cfg.stream = self.stream.cuda_stream
        self.cfg = cfg
        self.n_workers = int(n_workers)
        self._h = _vp()
        _check(lib().alsgd_init(C.byref(self._h), self.tab, len(self.tab), self.align, C.byref(cfg)), "alsgd_init")

    # -- views of borrowed device memory ---------------------------------------------------------
    def _view(self, ptr, dtype):
        if not ptr:
            return None
        torch = self.torch
        off = int(ptr) - self.arena.data_ptr()
        size = self.P * (2 if dtype in (torch.int16, torch.bfloat16) else 4)
        return self.arena[off:off + size].view(dtype)

    def alsgd_state_ptrs(self):
        """(theta, m, Delta) as fp32 torch views of the arena."""
        p = Ptrs()
        _check(lib().alsgd_state_ptrs(self._h, C.byref(p)), "alsgd_state_ptrs", self._h)
        f = self.torch.float32
        return self._view(p.theta, f), self._view(p.m, f), self._view(p.delta, f)

    def alsgd_worker_state_ptrs(self, w):
        """dict of torch views: p, base, adam_m, adam_v (fp32), replica (int16 bit patterns)."""
        p = WorkerPtrs()
        _check(lib().alsgd_worker_state_ptrs(self._h, int(w), C.byref(p)), "alsgd_worker_state_ptrs", self._h)
        f = self.torch.float32
        return {"p": self._view(p.p, f), "base": self._view(p.base, f), "adam_m": self._view(p.adam_m, f),
                "adam_v": self._view(p.adam_v, f), "replica": self._view(p.replica, self.torch.int16)}

    # -- the ABI calls ---------------------------------------------------------------------------------
    def _ptr(self, t):
        """(address, is_device) of a contiguous fp32 torch tensor or numpy array of P elements."""
        if hasattr(t, "data_ptr"):
            assert t.is_contiguous() and t.dtype == self.torch.float32 and t.numel() == self.P
            return t.data_ptr(), int(t.is_cuda)
        assert t.flags["C_CONTIGUOUS"] and t.dtype.name == "float32" and t.size == self.P
        return t.ctypes.data, 0

    def alsgd_set_global(self, src):
        a, d = self._ptr(src)
        _check(lib().alsgd_set_global(self._h, a, d), "alsgd_set_global", self._h)

    def alsgd_get_global(self, dst):
        a, d = self._ptr(dst)
        _check(lib().alsgd_get_global(self._h, a, d), "alsgd_get_global", self._h)

    def alsgd_set_worker_params(self, w, src):
        a, d = self._ptr(src)
        _check(lib().alsgd_set_worker_params(self._h, int(w), a, d), "alsgd_set_worker_params", self._h)

    def alsgd_get_worker_params(self, w, dst):
        a, d = self._ptr(dst)
        _check(lib().alsgd_get_worker_params(self._h, int(w), a, d), "alsgd_get_worker_params", self._h)

    def alsgd_pull(self, w):
        _check(lib().alsgd_pull(self._h, int(w)), "alsgd_pull", self._h)

    def alsgd_inner_adamw(self, w, grads, step, lr):
        a, d = self._ptr(grads)
        _check(lib().alsgd_inner_adamw(self._h, int(w), a, d, int(step), float(lr)), "alsgd_inner_adamw", self._h)

    @staticmethod
    def _infos(info, k):
        return [{"worker": int(i.worker), "tick": int(i.tick), "staleness": int(i.staleness),
                 "boundary": bool(i.boundary), "gnorm2": float(i.gnorm2), "nonfinite": int(i.nonfinite),
                 "dropped": bool(i.dropped)} for i in info[:k]]

    def alsgd_inner_adamw_bf16(self, w, grads, step, lr):
        """grads: contiguous torch tensor of P bf16 (or int16 bit patterns), on the device or pinned on the host."""
        assert grads.is_contiguous() and grads.numel() == self.P and grads.element_size() == 2
        _check(lib().alsgd_inner_adamw_bf16(self._h, int(w), grads.data_ptr(), int(grads.is_cuda), int(step), float(lr)),
               "alsgd_inner_adamw_bf16", self._h)

    def alsgd_arrive(self, worker_ids, flags=ARRIVE_RESEED, want_info=True):
        k = len(worker_ids)
        ids = (C.c_uint32 * max(k, 1))(*[int(x) for x in worker_ids])
        info = (ArrivalInfo * max(k, 1))() if want_info else None
        _check(lib().alsgd_arrive(self._h, ids, k, int(flags), info), "alsgd_arrive", self._h)
        return self._infos(info, k) if want_info else None

    def alsgd_arrive_ex(self, worker_ids, flags=ARRIVE_RESEED, weights=None, dc_lambda=0.0,
                        staleness_rule=STALE_NONE, stale_threshold=0, want_info=True):
        k = len(worker_ids)
        ids = (C.c_uint32 * max(k, 1))(*[int(x) for x in worker_ids])
        info = (ArrivalInfo * max(k, 1))() if want_info else None
        opts = ArriveOpts()
        wbuf = (C.c_float * max(k, 1))(*[float(x) for x in weights]) if weights is not None else None
        opts.weights = wbuf
        opts.dc_lambda, opts.staleness_rule, opts.stale_threshold = float(dc_lambda), int(staleness_rule), int(stale_threshold)
        _check(lib().alsgd_arrive_ex(self._h, ids, k, int(flags), C.byref(opts), info), "alsgd_arrive_ex", self._h)
        return self._infos(info, k) if want_info else None

    def alsgd_counters(self):
        t, ph = C.c_uint64(), C.c_uint32()
        _check(lib().alsgd_counters(self._h, C.byref(t), C.byref(ph)), "alsgd_counters", self._h)
        return int(t.value), int(ph.value)

    def alsgd_state_bytes(self):
        n = C.c_uint64()
        _check(lib().alsgd_state_bytes(self._h, C.byref(n)), "alsgd_state_bytes", self._h)
        return int(n.value)

    def alsgd_export_state(self):
        """The state image as a numpy uint8 array."""
        import numpy as np
        buf = np.empty(self.alsgd_state_bytes(), dtype=np.uint8)
        _check(lib().alsgd_export_state(self._h, buf.ctypes.data, buf.size), "alsgd_export_state", self._h)
        return buf

    def alsgd_import_state(self, image):
        assert image.dtype.name == "uint8" and image.flags["C_CONTIGUOUS"]
        _check(lib().alsgd_import_state(self._h, image.ctypes.data, image.size), "alsgd_import_state", self._h)

    def alsgd_sync(self):
        _check(lib().alsgd_sync(self._h), "alsgd_sync", self._h)

    def alsgd_debug_word_ptr(self):
        """Device address of the debug build's violation record (raises E_UNSUPPORTED on the normal build)."""
        out = _vp()
        _check(lib().alsgd_debug_word_ptr(self._h, C.byref(out)), "alsgd_debug_word_ptr", self._h)
        return int(out.value)

    def raw(self, name, *args):
        """Call an ABI function on this context and return its status without raising."""
        return getattr(lib(), name)(self._h, *args)

    def close(self):
        if self._h:
            lib().alsgd_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# -- training operators of the workers -----------------------------------------------------------------
def _dtype_code(torch, dtype):
    if dtype == torch.float32:
        return F32
    if dtype == torch.bfloat16:
        return BF16
    raise AlsgdError(E_ARG, f"unsupported type {dtype}")


def _whole_code(torch, dtype):
    if dtype == torch.int32:
        return I32
    if dtype == torch.int64:
        return I64
    raise AlsgdError(E_ARG, f"unsupported type {dtype}")


def _stream(torch, index, stream):
    """Raw handle of the given stream, or of the device's current one (without building a Stream object)."""
    return stream.cuda_stream if stream is not None else torch._C._cuda_getCurrentRawStream(index)


class _Workspace:
    """Device memory of a plan.  It belongs to the stream that it was made for, and a stream that uses it besides is told to
    the allocator: a plan may go while its last kernels still run, and the memory must not have another owner before them."""

    def __init__(self, torch, nbytes, device, stream, zeroed=False):
        # the default stream under its own name: under another the allocator kept nothing of it for the next plan
        self._stream_of = lambda raw: torch.cuda.ExternalStream(raw, device=device) if raw else torch.cuda.default_stream(device)
        make = lambda: (torch.zeros if zeroed else torch.empty)(nbytes + 256, dtype=torch.uint8, device=device)  # noqa: E731
        if stream == _stream(torch, device.index, None):
            self._bytes = make()
        else:
            with torch.cuda.stream(self._stream_of(stream)):
                self._bytes = make()
        self.ptr, self.nbytes = -(-self._bytes.data_ptr() // 256) * 256, nbytes
        self._streams = {stream}

    def used_on(self, stream):
        if stream not in self._streams:
            self._bytes.record_stream(self._stream_of(stream))
            self._streams.add(stream)


class GradClip:
    """Gradient clipping for one tensor table: keeps the sizes, offsets and types of the gradients and the call's
    workspace; the tensors themselves are given at every call."""

    def __init__(self, numels, offsets, dtypes, out_dtype, device=0):
        import torch
        self.torch = torch
        self.device = torch.device("cuda", device)
        n = len(numels)
        assert n == len(offsets) == len(dtypes)
        self.numels, self.dtypes = [int(x) for x in numels], list(dtypes)
        self.out_dtype, self._out_code = out_dtype, _dtype_code(torch, out_dtype)
        self._desc = (GradDesc * max(n, 1))()
        for d, numel, off, t in zip(self._desc, self.numels, offsets, self.dtypes):
            d.numel, d.offset, d.dtype = numel, int(off), _dtype_code(torch, t)
        # the descriptors' pointers as a strided array, so that a call fills them at once
        import numpy as np
        self._ptrs = np.frombuffer(self._desc, dtype=np.uint64).reshape(max(n, 1), C.sizeof(GradDesc) // 8)[:n, 0]
        self._dtype_of, self._index = operator.attrgetter("dtype"), int(device)
        # calls of several threads go out one by one: they share the descriptors and, in stream order, the workspace
        self._lock = threading.Lock()
        nbytes = C.c_uint64()
        _check(lib().alsgd_clip_grads_bytes(n, C.byref(nbytes)), "alsgd_clip_grads_bytes")
        self._work = _Workspace(torch, int(nbytes.value), self.device, _stream(torch, self._index, None), zeroed=True)
        # the zeros are there before any stream uses the workspace
        torch.cuda.current_stream(self.device).synchronize()

    def alsgd_clip_grads(self, grads, max_norm, out, stats, stream=None):
        """grads: one contiguous device tensor per table entry.  out: flat tensor of out_dtype, or None for the norm
        alone.  stats: two fp32 values on the device (norm, factor)."""
        T = self.torch.Tensor
        assert list(map(T.numel, grads)) == self.numels and list(map(self._dtype_of, grads)) == self.dtypes
        assert all(map(T.is_contiguous, grads)) and all(i == self._index for i in map(T.get_device, grads))
        assert stats.numel() == 2 and stats.dtype == self.torch.float32 and stats.get_device() == self._index and stats.is_contiguous()
        if out is not None:
            assert out.dtype == self.out_dtype and out.is_contiguous() and out.get_device() == self._index
        raw = _stream(self.torch, self._index, stream)
        with self._lock:
            self._ptrs[:] = list(map(T.data_ptr, grads))
            self._work.used_on(raw)
            _check(lib().alsgd_clip_grads(self._desc, len(self.numels), max_norm, out.data_ptr() if out is not None else None,
                                          self._out_code, out.numel() if out is not None else 0, stats.data_ptr(),
                                          self._work.ptr, self._work.nbytes, self._index, raw), "alsgd_clip_grads")


def alsgd_attn_status(device=0):
    """0, or bits of the waits inside the attention kernels that ran out on this device (waits for the device)."""
    out = C.c_uint32()
    _check(lib().alsgd_attn_status(int(device), C.byref(out)), "alsgd_attn_status")
    return int(out.value)


class Attention:
    """Attention of one shape.  Operands are bf16 tensors [batch, position, head, dim] with any strides the ABI takes."""

    def __init__(self, batch, len_q, len_kv, heads_q, heads_kv, dim, causal=True, scale=None, q_pos=None, buckets=0,
                 max_distance=128, bidirectional=False, table_dtype=None, device=0):
        import torch
        self.torch = torch
        self.device = torch.device("cuda", device)
        d = self.desc = AttnDesc()
        d.batch, d.heads_q, d.heads_kv, d.len_q, d.len_kv, d.dim = [int(x) for x in (batch, heads_q, heads_kv, len_q, len_kv, dim)]
        d.flags = (ATTN_CAUSAL if causal else 0) | (ATTN_BIAS_TWO_SIDED if bidirectional else 0)
        d.buckets, d.max_distance = int(buckets), int(max_distance)
        self.table_dtype = table_dtype if table_dtype is not None else torch.float32
        d.table_dtype = _dtype_code(torch, self.table_dtype)
        d.q_pos = int(len_kv - len_q if q_pos is None else q_pos)
        d.scale = float(dim ** -0.5 if scale is None else scale)
        d.device = int(device)
        self._q_shape, self._kv_shape = (batch, len_q, heads_q, dim), (batch, len_kv, heads_kv, dim)
        self._lse_shape, self._table_shape = (batch, heads_q, len_q), (heads_q, buckets)
        self._bf16, self._index = torch.bfloat16, int(device)
        self._work = None                  # of the backward pass, made at its first call
        self._lock = threading.Lock()      # its calls go out one by one: they share the workspace, in stream order

    def _operand(self, t, shape):
        assert t.dtype is self._bf16 and t.shape == shape and t.get_device() == self._index
        b, s, h, d = t.stride()
        assert d == 1
        return AttnTensor(t.data_ptr(), b, s, h)

    def _plain(self, t, shape, dtype):
        if t is None:
            return None
        assert t.dtype is dtype and t.shape == shape and t.get_device() == self._index and t.is_contiguous()
        return t.data_ptr()

    def alsgd_attn_fwd(self, q, k, v, out, lse, table=None, kv_len=None, stream=None):
        """out and lse are written.  table: [heads_q, buckets]; kv_len: int32 per sequence."""
        _check(lib().alsgd_attn_fwd(self.desc, self._operand(q, self._q_shape), self._operand(k, self._kv_shape),
                                    self._operand(v, self._kv_shape), self._plain(table, self._table_shape, self.table_dtype),
                                    self._plain(kv_len, self._q_shape[:1], self.torch.int32), self._operand(out, self._q_shape),
                                    self._plain(lse, self._lse_shape, self.torch.float32),
                                    _stream(self.torch, self._index, stream)), "alsgd_attn_fwd")

    def alsgd_attn_bwd(self, q, k, v, out, lse, dout, dq, dk, dv, table=None, dtable=None, kv_len=None, stream=None):
        """dq, dk, dv and dtable are written.  The workspace belongs to this object: calls on several streams must be
        ordered by the caller."""
        raw = _stream(self.torch, self._index, stream)
        operands = [self._operand(t, shape) for t, shape in (
            (q, self._q_shape), (k, self._kv_shape), (v, self._kv_shape), (out, self._q_shape), (dout, self._q_shape),
            (dq, self._q_shape), (dk, self._kv_shape), (dv, self._kv_shape))]
        plain = [self._plain(table, self._table_shape, self.table_dtype), self._plain(kv_len, self._q_shape[:1], self.torch.int32),
                 self._plain(lse, self._lse_shape, self.torch.float32), self._plain(dtable, self._table_shape, self.table_dtype)]
        with self._lock:
            if self._work is None:
                nbytes = C.c_uint64()
                _check(lib().alsgd_attn_bwd_bytes(self.desc, C.byref(nbytes)), "alsgd_attn_bwd_bytes")
                self._work = _Workspace(self.torch, int(nbytes.value), self.device, raw)
            self._work.used_on(raw)
            _check(lib().alsgd_attn_bwd(self.desc, *operands[:3], *plain[:2], operands[3], plain[2], *operands[4:], plain[3],
                                        self._work.ptr, self._work.nbytes, raw), "alsgd_attn_bwd")

    def alsgd_attn_bucket(self, distance):
        """Bucket of a distance key position - query position."""
        out = C.c_uint32()
        _check(lib().alsgd_attn_bucket(self.desc, int(distance), C.byref(out)), "alsgd_attn_bucket")
        return int(out.value)


def alsgd_vocab_status(device=0):
    """0, or bits of the waits inside the vocabulary kernels that ran out on this device (waits for the device)."""
    out = C.c_uint32()
    _check(lib().alsgd_vocab_status(int(device), C.byref(out)), "alsgd_vocab_status")
    return int(out.value)


class Rotary:
    """Rotary positions of one shape.  Operands are tensors [batch, position, head, dim] of `dtype` with any strides the ABI
    takes; `turns` = (turns_low, turns_high)."""

    def __init__(self, batch, length, heads_q, heads_k, dim, rot=None, interleaved=False, base=10000.0, factor=1.0, context=0.0,
                 turns=(0.0, 0.0), amplitude=1.0, pos0=0, dtype=None, device=0):
        import torch
        self.torch = torch
        self.dtype = dtype if dtype is not None else torch.bfloat16
        d = RopeDesc()
        d.batch, d.len, d.heads_q, d.heads_k, d.dim = [int(x) for x in (batch, length, heads_q, heads_k, dim)]
        d.rot = int(dim if rot is None else rot)
        d.flags = ROPE_INTERLEAVED if interleaved else 0
        d.dtype, d.position_dtype = _dtype_code(torch, self.dtype), I32
        d.pos0, d.device = int(pos0), int(device)
        d.base, d.factor, d.context, d.amplitude = float(base), float(factor), float(context), float(amplitude)
        d.turns_low, d.turns_high = float(turns[0]), float(turns[1])
        # a call's direction, the positions' type and which operands there are choose among descriptors, each made at its first call
        self._descs = {(False, I32, "both"): d}
        self._q_shape, self._k_shape = (batch, length, heads_q, dim), (batch, length, heads_k, dim)
        self._index = int(device)
        # filled at every call (making new ones costs as much again as all other checks), so calls go out one by one
        self._slots, self._lock = [AttnTensor() for _ in range(4)], threading.Lock()

    def _operand(self, slot, t, shape):
        assert t.dtype is self.dtype and t.shape == shape and t.get_device() == self._index
        slot.stride_batch, slot.stride_pos, slot.stride_head, d = t.stride()
        assert d == 1
        slot.data = t.data_ptr()
        return slot

    def _desc(self, inverse, code, which):
        d = self._descs.get((inverse, code, which))
        if d is None:
            d = RopeDesc.from_buffer_copy(self._descs[False, I32, "both"])
            d.flags |= ROPE_INVERSE if inverse else 0
            d.position_dtype = code
            d.heads_q, d.heads_k = {"both": (d.heads_q, d.heads_k), "q": (d.heads_q, 0), "k": (d.heads_k, 0)}[which]
            self._descs[inverse, code, which] = d
        return d

    def alsgd_rope(self, q, k, q_out, k_out, positions=None, inverse=False, stream=None):
        """q_out and k_out are written and may be q and k.  k and k_out are None without key heads or to turn q alone, q and q_out to
        turn k alone.  positions: int32 or int64 [batch, position]; inverse: the backward pass, on gradients."""
        code = I32
        if positions is not None:
            assert positions.shape == self._q_shape[:2] and positions.is_contiguous() and positions.get_device() == self._index
            code = _whole_code(self.torch, positions.dtype)
        assert (q is None) == (q_out is None) and (k is None) == (k_out is None)
        at = positions.data_ptr() if positions is not None else None
        q_in, k_in, q_to, k_to = self._slots
        shape, which = self._q_shape, "both"
        if k is None:
            which = "q"
        elif q is None:
            q, q_out, shape, which = k, k_out, self._k_shape, "k"
        with self._lock:
            self._operand(q_in, q, shape)
            self._operand(q_to, q_out, shape)
            if which == "both":
                self._operand(k_in, k, self._k_shape)
                self._operand(k_to, k_out, self._k_shape)
            _check(lib().alsgd_rope(self._desc(bool(inverse), code, which), q_in, k_in if which == "both" else None, at, q_to,
                                    k_to if which == "both" else None, _stream(self.torch, self._index, stream)), "alsgd_rope")

    def alsgd_rope_frequencies(self):
        """Angle per position of every pair, scaled as the plan says."""
        d = self._descs[False, I32, "both"]
        out = (C.c_double * (d.rot // 2))()
        _check(lib().alsgd_rope_frequencies(d, out), "alsgd_rope_frequencies")
        return [float(x) for x in out]


class VocabLoss:
    """Losses of `rows` rows over a vocabulary: labels (top = 0) or a teacher's `top` highest logits.  x: bf16 [rows, dim],
    w: bf16 [vocab, dim], rows any aligned distance apart.  The workspaces belong to this object: calls on several streams must
    be ordered by the caller."""

    def __init__(self, rows, vocab, dim, top=0, scale=1.0, index_dtype=None, teacher_dtype=None, device=0):
        import torch
        self.torch = torch
        self.device = torch.device("cuda", device)
        self.index_dtype = index_dtype if index_dtype is not None else torch.int64
        self.teacher_dtype = teacher_dtype if teacher_dtype is not None else torch.float32
        d = self.desc = VocabDesc()
        d.rows, d.vocab, d.dim, d.top, d.device = [int(x) for x in (rows, vocab, dim, top, device)]
        d.index_dtype, d.teacher_dtype, d.scale = _whole_code(torch, self.index_dtype), _dtype_code(torch, self.teacher_dtype), float(scale)
        self._x_shape, self._w_shape, self._rows = (rows, dim), (vocab, dim), (rows,)
        self._labels_shape = (rows, top) if top else (rows,)
        self._index = int(device)
        self._work = {}                    # of either pass, made at its first call
        self._slots = [Matrix() for _ in range(4)]
        # its calls go out one by one: they share the matrices' descriptors and, in stream order, the workspaces
        self._lock = threading.Lock()
        self._bf16, self._f32 = torch.bfloat16, torch.float32

    def _matrix(self, slot, t, shape):
        assert t.dtype is self._bf16 and t.shape == shape and t.get_device() == self._index
        slot.stride_row, d = t.stride()
        assert d == 1 or shape[1] == 1
        slot.data = t.data_ptr()
        return slot

    def _plain(self, t, shape, dtype):
        assert t.dtype is dtype and t.shape == shape and t.get_device() == self._index and t.is_contiguous()
        return t.data_ptr()

    def _workspace(self, backward, raw):
        work = self._work.get(backward)
        if work is None:
            nbytes = C.c_uint64()
            _check(lib().alsgd_vocab_bytes(self.desc, int(backward), C.byref(nbytes)), "alsgd_vocab_bytes")
            work = self._work[backward] = _Workspace(self.torch, int(nbytes.value), self.device, raw)
        work.used_on(raw)
        return work

    def _forward(self, name, x, w, labels, loss, lse, stream):
        raw = _stream(self.torch, self._index, stream)
        loss, lse = self._plain(loss, self._rows, self._f32), self._plain(lse, self._rows, self._f32)
        with self._lock:
            work, (sx, sw, _, _) = self._workspace(False, raw), self._slots
            _check(getattr(lib(), name)(self.desc, self._matrix(sx, x, self._x_shape), self._matrix(sw, w, self._w_shape), *labels, loss, lse,
                                        work.ptr, work.nbytes, raw), name)

    def _backward(self, name, x, w, labels, lse, dloss, dx, dw, stream):
        assert dloss.dtype is self._f32 and dloss.shape == self._rows and dloss.get_device() == self._index
        raw = _stream(self.torch, self._index, stream)
        lse = self._plain(lse, self._rows, self._f32)
        with self._lock:
            work, (sx, sw, sdx, sdw) = self._workspace(True, raw), self._slots
            _check(getattr(lib(), name)(self.desc, self._matrix(sx, x, self._x_shape), self._matrix(sw, w, self._w_shape), *labels, lse,
                                        dloss.data_ptr(), dloss.stride(0), self._matrix(sdx, dx, self._x_shape) if dx is not None else None,
                                        self._matrix(sdw, dw, self._w_shape) if dw is not None else None, work.ptr, work.nbytes, raw), name)

    def _labels(self, index):
        return (self._plain(index, self._labels_shape, self.index_dtype),)

    def _teacher(self, index, teacher):
        return self._labels(index) + (self._plain(teacher, self._labels_shape, self.teacher_dtype),)

    def alsgd_xent_fwd(self, x, w, target, loss, lse, stream=None):
        """loss and lse (fp32 [rows]) are written.  target: [rows]; a row whose target is no word takes no part."""
        self._forward("alsgd_xent_fwd", x, w, self._labels(target), loss, lse, stream)

    def alsgd_xent_bwd(self, x, w, target, lse, dloss, dx, dw, stream=None):
        """dx and dw are written, or the one that is not None.  dloss: fp32 [rows], which may be one number expanded."""
        self._backward("alsgd_xent_bwd", x, w, self._labels(target), lse, dloss, dx, dw, stream)

    def alsgd_distill_fwd(self, x, w, index, teacher, loss, lse, stream=None):
        """index, teacher: [rows, top], the teacher's words and logits; an entry whose index is no word takes no part."""
        self._forward("alsgd_distill_fwd", x, w, self._teacher(index, teacher), loss, lse, stream)

    def alsgd_distill_bwd(self, x, w, index, teacher, lse, dloss, dx, dw, stream=None):
        """dx and dw are written, or the one that is not None.  dloss: fp32 [rows], which may be one number expanded."""
        self._backward("alsgd_distill_bwd", x, w, self._teacher(index, teacher), lse, dloss, dx, dw, stream)
