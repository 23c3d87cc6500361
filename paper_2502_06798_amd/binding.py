"""Thin ctypes binding of libapc.so (include/apc.h), argument marshalling only.

Every function has the C name and takes torch tensors where the C call takes
device pointers; host tables are numpy arrays or sequences.  All compute runs
in the HIP library; when the library is missing this module raises instead of
falling back to anything else.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libapc.so")

APC_F32, APC_F16, APC_BF16, APC_E4M3 = 0, 1, 2, 3
STATUS = ("APC_OK", "APC_E_ARG", "APC_E_DTYPE", "APC_E_TABLE", "APC_E_NONFINITE",
          "APC_E_ZERO_NORM", "APC_E_WORKSPACE", "APC_E_NOMEM", "APC_E_HIP")
APC_MAX_K, APC_MAX_LEVELS, APC_MAX_INST = 64, 32, 256

DTYPE_OF = {torch.float32: APC_F32, torch.float16: APC_F16, torch.bfloat16: APC_BF16,
            torch.float8_e4m3fn: APC_E4M3}


class ApcError(RuntimeError):
    def __init__(self, status: int, msg: str):
        self.status = status
        self.name = STATUS[status] if 0 <= status < len(STATUS) else str(status)
        super().__init__(f"{self.name}: {msg}")


class _KvStruct(ctypes.Structure):
    """apc_kv of include/apc.h."""
    _fields_ = [("dt", ctypes.c_int), ("heads", ctypes.c_int32), ("d", ctypes.c_int32), ("page", ctypes.c_int32),
                ("n_pages", ctypes.c_int64), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


_lib = None


def load() -> ctypes.CDLL:
    """Load libapc.so (or the build APC_LIB names, e.g. one whose host code is
    instrumented by sanitizers); raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = os.environ.get("APC_LIB", "") or LIB_PATH
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with "
                          "`python -m paper_2502_06798_amd.build_lib` (hipcc, gfx950)")
    L = ctypes.CDLL(path)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    st = ctypes.c_int
    L.apc_build_cache.argtypes = [ctypes.c_int, i64, i32, vp, vp, vp, i64, i64, vp, vp,
                                  ctypes.POINTER(vp)]
    L.apc_build_cache.restype = st
    L.apc_destroy_cache.argtypes = [vp]
    L.apc_destroy_cache.restype = None
    L.apc_row_factors.argtypes = [ctypes.c_int, i64, i32, vp, vp, vp]
    L.apc_row_factors.restype = st
    L.apc_quantize_rows.argtypes = [ctypes.c_int, i64, i32, vp, vp, vp, vp]
    L.apc_quantize_rows.restype = st
    L.apc_validate_rows.argtypes = [ctypes.c_int, i64, i32, vp, vp, vp, ctypes.POINTER(i64), ctypes.POINTER(i64), vp]
    L.apc_validate_rows.restype = st
    L.apc_cache_row_factors.argtypes = [vp, vp, vp]
    L.apc_cache_row_factors.restype = st
    L.apc_match_workspace.argtypes = [vp, i32, i32, ctypes.POINTER(sz)]
    L.apc_match_workspace.restype = st
    L.apc_match_batch.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp, sz, vp]
    L.apc_match_batch.restype = st
    L.apc_match_batch_static.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp]
    L.apc_match_batch_static.restype = st
    L.apc_assign.argtypes = [vp, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.apc_assign.restype = st
    L.apc_assign_load_aware.argtypes = [vp, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp,
                                        vp, vp, vp]
    L.apc_assign_load_aware.restype = st
    L.apc_route_plan.argtypes = [i32, vp, vp, vp, vp, ctypes.POINTER(i64)]
    L.apc_route_plan.restype = st
    L.apc_assign_routed.argtypes = [vp, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.apc_assign_routed.restype = st
    L.apc_assign_planned.argtypes = [vp, i32, i32, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    L.apc_assign_planned.restype = st
    L.apc_resident_best.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp]
    L.apc_resident_best.restype = st
    L.apc_level_histogram.argtypes = [vp, i32, i32, vp, vp]
    L.apc_level_histogram.restype = st
    L.apc_gather_latents_at_level.argtypes = [vp, vp, i32, i32, vp, vp, vp, i32, i32, i32, vp, vp, vp]
    L.apc_gather_latents_at_level.restype = st
    L.apc_merge_shards.argtypes = [vp, vp, i32, i32, i32, vp, i32, vp, vp, vp]
    L.apc_merge_shards.restype = st
    L.apc_gather_latents.argtypes = [vp, vp, i32, i32, vp, vp, vp, i32, i32, vp, vp, vp]
    L.apc_gather_latents.restype = st
    f32, kv = ctypes.c_float, ctypes.POINTER(_KvStruct)
    L.apc_norm_rows.argtypes = [ctypes.c_int, ctypes.c_int, i64, i32, vp, i64, vp, i64, vp, f32, vp, i64, vp, i64, vp, vp]
    L.apc_norm_rows.restype = st
    L.apc_kv_write.argtypes = [kv, ctypes.c_int, i64, vp, i64, i64, vp, i64, i64, vp, vp]
    L.apc_kv_write.restype = st
    L.apc_kv_read.argtypes = [kv, ctypes.c_int, i64, vp, vp, i64, i64, vp, i64, i64, vp]
    L.apc_kv_read.restype = st
    L.apc_attend_workspace.argtypes = [kv, i32, i32, i32, ctypes.POINTER(sz)]
    L.apc_attend_workspace.restype = st
    L.apc_attend.argtypes = [kv, ctypes.c_int, vp, i64, i64, i32, i32, vp, i32, i64, vp, i32, f32, vp, i64, i64, vp, vp,
                             sz, vp]
    L.apc_attend.restype = st
    L.apc_set_kernel_events.argtypes = [vp, vp]
    L.apc_set_kernel_events.restype = st
    L.apc_status_str.argtypes = [ctypes.c_int]
    L.apc_status_str.restype = ctypes.c_char_p
    L.apc_last_error.argtypes = []
    L.apc_last_error.restype = ctypes.c_char_p
    _lib = L
    return L


def _check(rc: int):
    if rc != 0:
        raise ApcError(rc, load().apc_last_error().decode())


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    return ctypes.c_void_p(t.data_ptr())


# The current stream's handle without the Stream object that torch.cuda.current_stream() makes (2.7 us a call, 0.2 so).
_raw_stream, _device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> ctypes.c_void_p:
    if stream is None:
        if _raw_stream is not None and _device is not None:
            return ctypes.c_void_p(_raw_stream(_device()))
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _host(a, dtype) -> Optional[np.ndarray]:
    if a is None:
        return None
    return np.ascontiguousarray(np.asarray(a), dtype=dtype)


def _hp(a: Optional[np.ndarray]):
    return None if a is None else a.ctypes.data_as(ctypes.c_void_p)


def apc_status_str(status: int) -> str:
    return load().apc_status_str(status).decode()


def apc_last_error() -> str:
    return load().apc_last_error().decode()


def apc_set_kernel_events(start, stop):
    """start/stop: raw hipEvent_t handles (ints or c_void_p), or None, None."""
    _check(load().apc_set_kernel_events(start, stop))


class Cache:
    """Handle over a built cache; keeps the borrowed tensors alive."""

    def __init__(self, handle: ctypes.c_void_p, dtype: int, n: int, d: int, keep: tuple):
        self.handle = handle
        self.dtype, self.n, self.d = dtype, n, d
        self._keep = keep

    def close(self):
        if self.handle:
            torch.cuda.synchronize()
            load().apc_destroy_cache(self.handle)
            self.handle = None

    def __del__(self):
        try:
            if self.handle and _lib is not None:
                _lib.apc_destroy_cache(self.handle)
                self.handle = None
        except Exception:
            pass


def apc_build_cache(emb: torch.Tensor, row_scale: Optional[torch.Tensor] = None,
                    latents: Optional[torch.Tensor] = None,
                    slot_of_entry: Optional[torch.Tensor] = None, stream=None) -> Cache:
    """emb: n x d device tensor (float32/float16/bfloat16/float8_e4m3fn);
    latents: n_slots x latent_bytes uint8 device tensor or None."""
    L = load()
    if emb.dim() != 2 or emb.dtype not in DTYPE_OF:
        raise ValueError("emb must be a 2-D float32/float16/bfloat16/float8_e4m3fn tensor")
    n, d = emb.shape
    n_slots, lb = (0, 0) if latents is None else (latents.shape[0], latents[0].numel() * latents.element_size())
    out = ctypes.c_void_p()
    _check(L.apc_build_cache(DTYPE_OF[emb.dtype], n, d, _ptr(emb), _ptr(row_scale), _ptr(latents),
                             n_slots, lb, _ptr(slot_of_entry), _stream(stream), ctypes.byref(out)))
    return Cache(out, DTYPE_OF[emb.dtype], n, d, (emb, row_scale, latents, slot_of_entry))


def apc_destroy_cache(c: Cache):
    c.close()


def apc_row_factors(rows: torch.Tensor, out: torch.Tensor, stream=None):
    n, d = rows.shape
    _check(load().apc_row_factors(DTYPE_OF[rows.dtype], n, d, _ptr(rows), _ptr(out), _stream(stream)))


def apc_quantize_rows(x: torch.Tensor, out: torch.Tensor, row_scale=None, stream=None):
    """float32 rows x into out (f16, bf16 or e4m3fn; row_scale for e4m3fn)."""
    n, d = x.shape
    _check(load().apc_quantize_rows(DTYPE_OF[out.dtype], n, d, _ptr(x), _ptr(out), _ptr(row_scale), _stream(stream)))


def apc_validate_rows(rows: torch.Tensor, row_scale=None, bad=None, stream=None):
    """(bad-row count, lowest bad row or -1); per-row flags into bad (uint8) if given."""
    n, d = rows.shape
    nb, fb = ctypes.c_int64(), ctypes.c_int64()
    _check(load().apc_validate_rows(DTYPE_OF[rows.dtype], n, d, _ptr(rows), _ptr(row_scale), _ptr(bad),
                                    ctypes.byref(nb), ctypes.byref(fb), _stream(stream)))
    return nb.value, fb.value


def apc_cache_row_factors(c: Cache, out: torch.Tensor, stream=None):
    _check(load().apc_cache_row_factors(c.handle, _ptr(out), _stream(stream)))


def apc_match_workspace(c: Cache, b: int, k: int) -> int:
    n = ctypes.c_size_t()
    _check(load().apc_match_workspace(c.handle, b, k, ctypes.byref(n)))
    return n.value


def workspace_tensor(c: Cache, b: int, k: int, device=None) -> torch.Tensor:
    """Device buffer of apc_match_workspace() bytes (torch allocations are 256-byte aligned)."""
    return torch.empty(max(apc_match_workspace(c, b, k), 256), dtype=torch.uint8, device=device or "cuda")


def apc_match_batch(c: Cache, q: torch.Tensor, q_scale: Optional[torch.Tensor], k: int,
                    top_score: torch.Tensor, top_idx: torch.Tensor, ws: torch.Tensor, stream=None):
    b = q.shape[0]
    _check(load().apc_match_batch(c.handle, _ptr(q), _ptr(q_scale), b, k, _ptr(top_score),
                                  _ptr(top_idx), _ptr(ws), ws.numel() * ws.element_size(),
                                  _stream(stream)))


def apc_match_batch_static(c: Cache, q: torch.Tensor, q_scale: Optional[torch.Tensor], k: int,
                           top_score: torch.Tensor, top_idx: torch.Tensor, stream=None):
    """apc_match_batch on the library's static device workspace (allocates nothing)."""
    b = q.shape[0]
    _check(load().apc_match_batch_static(c.handle, _ptr(q), _ptr(q_scale), b, k, _ptr(top_score),
                                         _ptr(top_idx), _stream(stream)))


def apc_assign(top_score: torch.Tensor, ld: int, b: int, theta: Sequence[float], K: Sequence[int],
               inst_level: Sequence[int], inst_cap: Sequence[int], inst_queue: Optional[Sequence[int]],
               opt_level: torch.Tensor, out_level: torch.Tensor, out_inst: torch.Tensor,
               out_slot: torch.Tensor, inst_fill: torch.Tensor, stream=None):
    th = _host(theta, np.float32)
    Kh = _host(K, np.int32)
    il = _host(inst_level, np.int32)
    ic = _host(inst_cap, np.int32)
    iq = _host(inst_queue, np.int32)
    _check(load().apc_assign(_ptr(top_score), ld, b, th.size, _hp(th), _hp(Kh), il.size, _hp(il),
                             _hp(ic), _hp(iq), _ptr(opt_level), _ptr(out_level), _ptr(out_inst),
                             _ptr(out_slot), _ptr(inst_fill), _stream(stream)))


def apc_assign_load_aware(top_score: torch.Tensor, ld: int, b: int, theta: Sequence[float], K: Sequence[int],
                          inst_level: Sequence[int], inst_cap: Sequence[int], inst_queue: Optional[Sequence[int]],
                          inst_rand: Optional[Sequence[int]], load_value: int, load_threshold: int,
                          opt_level: torch.Tensor, out_level: torch.Tensor, out_inst: torch.Tensor,
                          out_slot: torch.Tensor, inst_fill: torch.Tensor, stream=None) -> int:
    """load_value: the caller's load measure (the C call's `load`).  Returns the
    routing used: 1 greedy, 0 uniform."""
    th = _host(theta, np.float32)
    Kh = _host(K, np.int32)
    il = _host(inst_level, np.int32)
    ic = _host(inst_cap, np.int32)
    iq = _host(inst_queue, np.int32)
    ir = _host(inst_rand, np.uint32)
    routing = ctypes.c_int32(-1)
    _check(load().apc_assign_load_aware(_ptr(top_score), ld, b, th.size, _hp(th), _hp(Kh), il.size, _hp(il),
                                        _hp(ic), _hp(iq), _hp(ir), int(load_value), int(load_threshold),
                                        ctypes.byref(routing), _ptr(opt_level), _ptr(out_level), _ptr(out_inst),
                                        _ptr(out_slot), _ptr(inst_fill), _stream(stream)))
    return routing.value


def apc_route_plan(K: Sequence[int], H: Sequence[int], F: Sequence[int]):
    """Host-only Route-Plan: returns (X as an (L+1) x (L+1) int32 array, degradation)."""
    Kh = _host(K, np.int32)
    Hh = _host(H, np.int32)
    Fh = _host(F, np.int32)
    L = Kh.size
    if Hh.size != L + 1 or Fh.size != L + 1:
        raise ValueError("apc_route_plan: H and F need len(K) + 1 entries")
    X = np.zeros((L + 1, L + 1), dtype=np.int32)
    d = ctypes.c_int64(0)
    _check(load().apc_route_plan(L, _hp(Kh), _hp(Hh), _hp(Fh), X.ctypes.data, ctypes.byref(d)))
    return X, int(d.value)


def _assign_plan(fn, top_score, ld, b, theta, K, inst_level, inst_cap, inst_queue, plan, opt_level,
                 out_level, out_inst, out_slot, inst_fill, stream):
    th = _host(theta, np.float32)
    Kh = _host(K, np.int32)
    il = _host(inst_level, np.int32)
    ic = _host(inst_cap, np.int32)
    iq = _host(inst_queue, np.int32)
    _check(fn(_ptr(top_score), ld, b, th.size, _hp(th), _hp(Kh), il.size, _hp(il), _hp(ic), _hp(iq),
              _ptr(plan), _ptr(opt_level), _ptr(out_level), _ptr(out_inst), _ptr(out_slot),
              _ptr(inst_fill), _stream(stream)))


def apc_assign_routed(top_score: torch.Tensor, ld: int, b: int, theta: Sequence[float], K: Sequence[int],
                      inst_level: Sequence[int], inst_cap: Sequence[int], inst_queue: Optional[Sequence[int]],
                      plan: torch.Tensor, opt_level: torch.Tensor, out_level: torch.Tensor,
                      out_inst: torch.Tensor, out_slot: torch.Tensor, inst_fill: torch.Tensor, stream=None):
    _assign_plan(load().apc_assign_routed, top_score, ld, b, theta, K, inst_level, inst_cap, inst_queue,
                 plan, opt_level, out_level, out_inst, out_slot, inst_fill, stream)


def apc_assign_planned(top_score: torch.Tensor, ld: int, b: int, theta: Sequence[float], K: Sequence[int],
                       inst_level: Sequence[int], inst_cap: Sequence[int], inst_queue: Optional[Sequence[int]],
                       plan: torch.Tensor, opt_level: torch.Tensor, out_level: torch.Tensor,
                       out_inst: torch.Tensor, out_slot: torch.Tensor, inst_fill: torch.Tensor, stream=None):
    _assign_plan(load().apc_assign_planned, top_score, ld, b, theta, K, inst_level, inst_cap, inst_queue,
                 plan, opt_level, out_level, out_inst, out_slot, inst_fill, stream)


def apc_resident_best(c: Cache, top_score: torch.Tensor, top_idx: torch.Tensor, ld: int, k: int, b: int,
                      out_score: torch.Tensor, out_idx: torch.Tensor, stream=None):
    _check(load().apc_resident_best(c.handle, _ptr(top_score), _ptr(top_idx), ld, k, b, _ptr(out_score),
                                    _ptr(out_idx), _stream(stream)))


def apc_level_histogram(level: torch.Tensor, b: int, L: int, hist: torch.Tensor, stream=None):
    _check(load().apc_level_histogram(_ptr(level), b, L, _ptr(hist), _stream(stream)))


def apc_gather_latents(c: Cache, top_idx: torch.Tensor, ld: int, b: int, out_level: torch.Tensor,
                       out_inst: torch.Tensor, out_slot: torch.Tensor, n_inst: int,
                       slots_per_inst: int, batch_latents: torch.Tensor, hit: torch.Tensor,
                       stream=None):
    _check(load().apc_gather_latents(c.handle, _ptr(top_idx), ld, b, _ptr(out_level), _ptr(out_inst),
                                     _ptr(out_slot), n_inst, slots_per_inst, _ptr(batch_latents),
                                     _ptr(hit), _stream(stream)))


def apc_gather_latents_at_level(c: Cache, top_idx: torch.Tensor, ld: int, b: int, out_level: torch.Tensor,
                                out_inst: torch.Tensor, out_slot: torch.Tensor, n_inst: int, slots_per_inst: int,
                                levels_per_slot: int, batch_latents: torch.Tensor, hit: torch.Tensor, stream=None):
    _check(load().apc_gather_latents_at_level(c.handle, _ptr(top_idx), ld, b, _ptr(out_level), _ptr(out_inst),
                                              _ptr(out_slot), n_inst, slots_per_inst, levels_per_slot,
                                              _ptr(batch_latents), _ptr(hit), _stream(stream)))


def apc_merge_shards(scores: torch.Tensor, idx: torch.Tensor, g: int, b: int, k_in: int, offsets: Sequence[int],
                     k: int, out_score: torch.Tensor, out_idx: torch.Tensor, stream=None):
    off = _host(offsets, np.int32)
    if off is None or off.size != g:
        raise ValueError("apc_merge_shards: need one offset per shard")
    _check(load().apc_merge_shards(_ptr(scores), _ptr(idx), g, b, k_in, _hp(off), k, _ptr(out_score),
                                   _ptr(out_idx), _stream(stream)))


# ---- operators of the prompt model ----

def _view(t: torch.Tensor, what: str, shape, dtype):
    """(address, strides) of a device tensor of that shape and type whose last axis is contiguous."""
    if t.shape != shape or t.dtype != dtype:
        raise ValueError(f"{what}: expected {dtype} of shape {tuple(shape)}, got {t.dtype} of {tuple(t.shape)}")
    if not t.is_cuda:
        raise ValueError(f"{what}: expected a device tensor")
    strides = t.stride()
    if strides[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{what}: the last axis must be contiguous")
    return t.data_ptr(), strides


def _dtype(t: torch.Tensor, what: str) -> int:
    dt = DTYPE_OF.get(t.dtype)
    if dt is None:
        raise ValueError(f"{what}: {t.dtype} is none of the library's types")
    return dt


def apc_norm_rows(x: torch.Tensor, out: torch.Tensor, weight: Optional[torch.Tensor] = None,
                  res: Optional[torch.Tensor] = None, sum_out: Optional[torch.Tensor] = None,
                  out_scale: Optional[torch.Tensor] = None, eps: float = 1e-6, stream=None):
    """Root-mean-square norm of the rows of x (+ res): n x d tensors whose rows may be strided.  out is of x's type
    or float8_e4m3fn (then out_scale holds a float32 scale per row); sum_out, if given, gets x + res."""
    shape, dtype = x.shape, x.dtype
    if len(shape) != 2:
        raise ValueError("x must be a 2-D tensor")
    n, d = shape
    dt, odt = _dtype(x, "x"), _dtype(out, "out")
    xp, xs = _view(x, "x", shape, dtype)
    op, os_ = _view(out, "out", shape, out.dtype)
    wp = rp = sp = cp = None
    rl = sl = d
    if weight is not None:
        wp, _ = _view(weight, "weight", (d,), dtype)
    if res is not None:
        rp, st = _view(res, "res", shape, dtype)
        rl = st[0] if n > 1 else d              # of one row, torch's row stride may be anything
    if sum_out is not None:
        sp, st = _view(sum_out, "sum_out", shape, dtype)
        sl = st[0] if n > 1 else d
    if out_scale is not None:
        cp, _ = _view(out_scale, "out_scale", (n,), torch.float32)
    rc = load().apc_norm_rows(dt, odt, n, d, xp, xs[0] if n > 1 else d, rp, rl, wp, eps, sp, sl, op,
                              os_[0] if n > 1 else d, cp, _stream(stream))
    if rc:
        _check(rc)


class KvCache:
    """Paged key-value cache over caller tensors: k and v n_pages x heads x page x d (float16, bfloat16 or
    float8_e4m3fn), k_scale and v_scale n_pages x heads x page float32 (float8_e4m3fn only).  Keeps the tensors
    alive; slot p * page + t is token t of page p."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        if k.dim() != 4:
            raise ValueError("k must be an n_pages x heads x page x d tensor")
        for t, what, shape, dtype in ((v, "v", k.shape, k.dtype), (k_scale, "k_scale", k.shape[:3], torch.float32),
                                      (v_scale, "v_scale", k.shape[:3], torch.float32)):
            if t is not None and (t.shape != shape or t.dtype != dtype):
                raise ValueError(f"{what}: expected {dtype} of shape {tuple(shape)}, got {t.dtype} of {tuple(t.shape)}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.heads, self.page, self.d = k.shape
        self.struct = _KvStruct(_dtype(k, "k"), self.heads, self.d, self.page, self.n_pages, _ptr(k), _ptr(v),
                                _ptr(k_scale), _ptr(v_scale))
        self.ref = ctypes.byref(self.struct)


def _kv_rows(c: KvCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor):
    if slots.dim() != 1:
        raise ValueError("slots must be a 1-D int32 tensor")
    t = slots.shape[0]
    shape, dtype = (t, c.heads, c.d), k.dtype
    kp, ks = _view(k, "k", shape, dtype)
    vp, vs = _view(v, "v", shape, dtype)
    sp, ss = _view(slots, "slots", (t,), torch.int32)
    return _dtype(k, "k"), t, kp, ks[0], ks[1], vp, vs[0], vs[1], sp


def apc_kv_write(c: KvCache, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, stream=None):
    """Keys and values (t x heads x d, tokens and heads strided as they come) into the cache's slots: each slot once,
    or outside the cache (-1), where nothing is written."""
    dt, t, kp, kt, kh, vp, vt, vh, sp = _kv_rows(c, k, v, slots)
    rc = load().apc_kv_write(c.ref, dt, t, kp, kt, kh, vp, vt, vh, sp, _stream(stream))
    if rc:
        _check(rc)


def apc_kv_read(c: KvCache, slots: torch.Tensor, k: torch.Tensor, v: torch.Tensor, stream=None):
    """The slots' keys and values into k and v (t x heads x d)."""
    dt, t, kp, kt, kh, vp, vt, vh, sp = _kv_rows(c, k, v, slots)
    rc = load().apc_kv_read(c.ref, dt, t, sp, kp, kt, kh, vp, vt, vh, _stream(stream))
    if rc:
        _check(rc)


def apc_attend_workspace(c: KvCache, b: int, q_heads: int, max_pages: int) -> int:
    n = ctypes.c_size_t()
    _check(load().apc_attend_workspace(c.ref, b, q_heads, max_pages, ctypes.byref(n)))
    return n.value


def attend_workspace_tensor(c: KvCache, b: int, q_heads: int, max_pages: int, device=None) -> torch.Tensor:
    """Device buffer of apc_attend_workspace() bytes (torch allocations are 256-byte aligned)."""
    return torch.empty(max(apc_attend_workspace(c, b, q_heads, max_pages), 256), dtype=torch.uint8,
                       device=device or "cuda")


def apc_attend(c: KvCache, q: torch.Tensor, pages: torch.Tensor, lengths: torch.Tensor, scale: float,
               out: torch.Tensor, ws: torch.Tensor, lse: Optional[torch.Tensor] = None, window: int = 0, stream=None):
    """Attention of one new token per sequence: q and out b x q_heads x d, pages b x max_pages int32 (page numbers of
    each sequence, rows may be strided), lengths b int32, lse b x q_heads float32 or None."""
    shape, dtype = q.shape, q.dtype
    if len(shape) != 3 or pages.dim() != 2:
        raise ValueError("q must be a b x q_heads x d tensor and pages a b x max_pages int32 tensor")
    b, q_heads, d = shape
    max_pages = pages.shape[1]
    if d != c.d:
        raise ValueError(f"q has {d} elements a head and the cache {c.d}")
    qp, qs = _view(q, "q", shape, dtype)
    op, os_ = _view(out, "out", shape, dtype)
    pp, ps = _view(pages, "pages", (b, max_pages), torch.int32)
    lp, _ = _view(lengths, "lengths", (b,), torch.int32)
    ep = None
    if lse is not None:
        if not lse.is_contiguous():
            raise ValueError("lse: expected a contiguous tensor")
        ep, _ = _view(lse, "lse", (b, q_heads), torch.float32)
    rc = load().apc_attend(c.ref, _dtype(q, "q"), qp, qs[0], qs[1], b, q_heads, pp, max_pages,
                           ps[0] if b > 1 else max_pages, lp, window, scale, op, os_[0], os_[1], ep, _ptr(ws),
                           ws.numel() * ws.element_size(), _stream(stream))
    if rc:
        _check(rc)
