"""Thin ctypes binding over libspd.so: same names as the C ABI, argument marshalling only.

PyTorch supplies device memory and streams; every step of the path runs in the library's
kernels.  There is no fallback: if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Tuple

import torch

from .build import LIB_PATH

SPD_OK = 0
SPD_F32, SPD_BF16 = 0, 1
SPD_PLAN_PER_CALL, SPD_PLAN_STORE, SPD_PLAN_REUSE = 0, 1, 2
_STATUS_NAMES = {0: "SPD_OK", 1: "SPD_ERR_INVALID_ARG", 2: "SPD_ERR_UNSUPPORTED", 3: "SPD_ERR_WORKSPACE",
                 4: "SPD_ERR_BAD_PAGE", 5: "SPD_ERR_CUDA", 6: "SPD_ERR_TIMEOUT", 7: "SPD_ERR_PLAN", 8: "SPD_ERR_NO_PAGE"}
_DEVICE_CODES = (SPD_OK, 4, 6, 7)     # what a call that waits for the device may report without raising

EXPORTS = ["spd_workspace_size", "spd_partial_attn", "spd_service_attn_merge", "spd_decode_step",
           "spd_step_blob_layout", "spd_decode_step_host", "spd_query_device_status",
           "spd_kernel_launch_count", "spd_status_string", "spd_profile_begin", "spd_profile_end",
           "spd_decode_step_static", "spd_append_kv",
           "spd_partial_attn_watch", "spd_decode_step_watch", "spd_set_bf16_math", "spd_merge_partials", "spd_prefill_attn",
           "spd_set_prefill_rows", "spd_token_step", "spd_partial_attn_planned", "spd_service_attn_merge_planned",
           "spd_decode_step_planned", "spd_set_split", "spd_set_programmatic_launch", "spd_debug_read_plan",
           "spd_debug_sm_moves", "spd_decode_step_append", "spd_watch_alarm", "spd_service_attn_merge_append",
           "spd_partial_attn_scored", "spd_service_attn_merge_scored", "spd_decode_step_scored", "spd_prefill_attn_scored",
           "spd_append_kv_rope", "spd_drafted_workspace_size", "spd_decode_step_drafted", "spd_partial_attn_drafted",
           "spd_service_attn_merge_drafted", "spd_keep_drafted", "spd_pages_workspace_size", "spd_pages_take", "spd_pages_release", "spd_pages_fork", "spd_pages_copy"]


class SpdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {_STATUS_NAMES.get(code, code)} ({status_string(code)})")


class Shape(C.Structure):
    _fields_ = [("batch", C.c_int32), ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("page_size", C.c_int32), ("dtype", C.c_int32), ("sm_scale", C.c_float)]


class PagedKV(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("num_pages", C.c_int32),
                ("page_indptr", C.c_void_p), ("page_indices", C.c_void_p), ("seq_lens", C.c_void_p)]


class Layer(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k_new", C.c_void_p), ("v_new", C.c_void_p), ("priv", PagedKV), ("pub", PagedKV),
                ("out", C.c_void_p)]


class StepBlob(C.Structure):
    _fields_ = [("priv_pages_listed", C.c_int64), ("pub_pages_listed", C.c_int64), ("q", C.c_size_t),
                ("priv_indptr", C.c_size_t), ("priv_lens", C.c_size_t), ("priv_indices", C.c_size_t),
                ("pub_indptr", C.c_size_t), ("pub_lens", C.c_size_t), ("pub_indices", C.c_size_t),
                ("status", C.c_size_t), ("in_bytes", C.c_size_t), ("out", C.c_size_t), ("total_bytes", C.c_size_t)]


class Watch(C.Structure):
    _fields_ = [("tok_lo", C.c_void_p), ("tok_hi", C.c_void_p), ("out", C.c_void_p)]


class Score(C.Structure):
    _fields_ = [("logit_cap", C.c_float), ("window", C.c_int32), ("alibi_slopes", C.c_void_p)]


class Tokens(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64),
                ("v_stride", C.c_int64)]


_Sections = C.c_int32 * 4


class Rope(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("interleaved", C.c_int32), ("num_axes", C.c_int32), ("sections", _Sections),
                ("scale", C.c_float), ("inv_freq", C.c_void_p)]


class Drafts(C.Structure):
    _fields_ = [("total_tokens", C.c_int64), ("tok_indptr", C.c_void_p), ("parents", C.c_void_p), ("sinks", C.c_int32)]


class Partial(C.Structure):
    _fields_ = [("o", C.c_void_p), ("m", C.c_void_p), ("l", C.c_void_p)]


_lib = None


def lib() -> C.CDLL:
    """Load libspd.so (built in-tree by build.py).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} not built: run `python -m paper_2409_19134_b200.build`")
        L = C.CDLL(LIB_PATH)
        vp, sz = C.c_void_p, C.c_size_t
        L.spd_workspace_size.argtypes = [C.POINTER(Shape), C.POINTER(sz)]
        L.spd_partial_attn.argtypes = [C.POINTER(Shape), vp, C.POINTER(PagedKV), Partial, vp, sz, vp]
        L.spd_service_attn_merge.argtypes = [C.POINTER(Shape), vp, C.POINTER(PagedKV), Partial, vp, C.c_int, vp, sz, vp]
        L.spd_decode_step.argtypes = [C.POINTER(Shape), vp, C.POINTER(PagedKV), C.POINTER(PagedKV), vp, C.c_int,
                                      C.c_int32, vp, sz, vp]
        L.spd_step_blob_layout.argtypes = [C.POINTER(Shape), C.c_int64, C.c_int64, C.c_int, C.POINTER(StepBlob)]
        L.spd_decode_step_host.argtypes = [C.POINTER(Shape), C.POINTER(StepBlob), vp, vp, C.POINTER(PagedKV),
                                           C.POINTER(PagedKV), C.c_int, C.POINTER(C.c_int32), vp, sz, vp]
        L.spd_query_device_status.argtypes = [vp, vp, C.POINTER(C.c_int32)]
        L.spd_kernel_launch_count.restype = C.c_int64
        L.spd_status_string.restype = C.c_char_p
        L.spd_status_string.argtypes = [C.c_int]
        L.spd_profile_begin.argtypes = [C.c_int32]
        L.spd_profile_end.argtypes = [C.POINTER(C.c_int32), C.POINTER(C.c_double)]
        L.spd_decode_step_static.argtypes = [C.POINTER(Shape), vp, C.POINTER(PagedKV), C.POINTER(PagedKV), vp, C.c_int,
                                             C.c_int32, C.POINTER(C.c_int32), vp]
        L.spd_partial_attn_watch.argtypes = [C.POINTER(Shape), vp, C.POINTER(PagedKV), Partial, C.POINTER(Watch), vp, sz, vp]
        L.spd_decode_step_watch.argtypes = [C.POINTER(Shape), vp, C.POINTER(PagedKV), C.POINTER(PagedKV), vp, C.c_int,
                                            C.POINTER(Watch), vp, sz, vp]
        L.spd_set_bf16_math.argtypes = [C.c_int32]
        L.spd_set_prefill_rows.argtypes = [C.c_int32]
        L.spd_token_step.argtypes = [C.POINTER(Shape), C.c_int32, C.POINTER(Layer), C.c_int, C.c_int32, vp, sz, vp]
        L.spd_partial_attn_planned.argtypes = [C.POINTER(Shape), vp, C.POINTER(PagedKV), Partial, C.c_int, vp, sz, vp]
        L.spd_service_attn_merge_planned.argtypes = [C.POINTER(Shape), vp, C.POINTER(PagedKV), Partial, vp, C.c_int, C.c_int,
                                                     vp, sz, vp]
        L.spd_decode_step_planned.argtypes = [C.POINTER(Shape), vp, C.POINTER(PagedKV), C.POINTER(PagedKV), vp, C.c_int,
                                              C.c_int32, C.c_int, vp, sz, vp]
        L.spd_decode_step_append.argtypes = [C.POINTER(Shape), vp, vp, vp, C.POINTER(PagedKV), C.POINTER(PagedKV), vp, C.c_int,
                                             C.c_int, vp, sz, vp]
        L.spd_service_attn_merge_append.argtypes = [C.POINTER(Shape), vp, vp, vp, C.POINTER(PagedKV), Partial, vp, C.c_int, C.c_int,
                                                    vp, sz, vp]
        L.spd_partial_attn_scored.argtypes = [C.POINTER(Shape), C.POINTER(Score), vp, C.POINTER(PagedKV), vp, Partial, C.c_int,
                                              vp, sz, vp]
        L.spd_service_attn_merge_scored.argtypes = [C.POINTER(Shape), C.POINTER(Score), vp, C.POINTER(PagedKV), vp, Partial, vp,
                                                    C.c_int, C.c_int, vp, sz, vp]
        L.spd_decode_step_scored.argtypes = [C.POINTER(Shape), C.POINTER(Score), vp, C.POINTER(PagedKV), C.POINTER(PagedKV), vp,
                                             C.c_int, C.c_int, vp, sz, vp]
        L.spd_prefill_attn_scored.argtypes = [C.POINTER(Shape), C.POINTER(Score), C.c_int64, C.POINTER(Tokens), vp, vp, vp, vp,
                                              C.c_int, vp, sz, vp]
        L.spd_append_kv_rope.argtypes = [C.POINTER(Shape), C.POINTER(Rope), C.c_int64, C.POINTER(Tokens), vp, vp, vp, vp, vp, vp,
                                         vp, C.c_int32, vp, vp, vp, vp, vp, sz, vp]
        L.spd_drafted_workspace_size.argtypes = [C.POINTER(Shape), C.POINTER(sz)]
        L.spd_decode_step_drafted.argtypes = [C.POINTER(Shape), C.POINTER(Score), C.POINTER(Drafts), vp, C.POINTER(PagedKV), C.POINTER(PagedKV),
                                              vp, C.c_int, vp, sz, vp]
        L.spd_partial_attn_drafted.argtypes = [C.POINTER(Shape), C.POINTER(Score), C.POINTER(Drafts), vp, C.POINTER(PagedKV), vp, Partial,
                                               vp, sz, vp]
        L.spd_service_attn_merge_drafted.argtypes = [C.POINTER(Shape), C.POINTER(Score), C.POINTER(Drafts), vp, C.POINTER(PagedKV), vp,
                                                     Partial, vp, C.c_int, vp, sz, vp]
        L.spd_keep_drafted.argtypes = [C.POINTER(Shape), C.c_int64, vp, vp, vp, C.c_int32, vp, C.c_int32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.spd_pages_workspace_size.argtypes = [C.POINTER(Shape), C.c_int32, C.POINTER(sz)]
        for name in ("take", "release"):
            getattr(L, "spd_pages_" + name).argtypes = [C.POINTER(Shape), C.c_int32, vp, vp, vp, vp, vp, vp, sz, vp]
        L.spd_pages_fork.argtypes = [C.POINTER(Shape), C.c_int32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.spd_pages_copy.argtypes = [C.POINTER(Shape), C.c_int32, vp, C.c_int32, C.c_int32, vp, vp, sz, vp]
        L.spd_watch_alarm.argtypes = [vp, C.c_int32, C.c_int32, vp, C.c_float, vp, vp]
        L.spd_set_split.argtypes = [C.c_int32, C.c_int32]
        L.spd_set_programmatic_launch.argtypes = [C.c_int32]
        L.spd_debug_read_plan.argtypes = [vp, C.c_int32, vp, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                          C.POINTER(C.c_int32), C.c_int32]
        L.spd_debug_sm_moves.argtypes = [vp, vp, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        L.spd_merge_partials.argtypes = [C.POINTER(Shape), C.c_int32, C.POINTER(Partial), vp, C.c_int, vp]
        L.spd_prefill_attn.argtypes = [C.POINTER(Shape), C.c_int64, vp, vp, vp, vp, vp, vp, C.c_int32, vp, vp, vp, vp,
                                       C.c_int, vp, sz, vp]
        L.spd_append_kv.argtypes = [C.POINTER(Shape), vp, vp, vp, vp, C.c_int32, vp, vp, vp, vp, sz, vp]
        for name in EXPORTS[:7] + EXPORTS[9:]:
            getattr(L, name).restype = C.c_int
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().spd_status_string(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != SPD_OK:
        raise SpdError(code, where)


def _dtype_code(dt: torch.dtype) -> int:
    if dt == torch.float32:
        return SPD_F32
    if dt == torch.bfloat16:
        return SPD_BF16
    raise TypeError(f"unsupported dtype {dt}")


def make_shape(batch, num_q_heads, num_kv_heads, head_dim, dtype, sm_scale, page_size=16) -> Shape:
    return Shape(batch, num_q_heads, num_kv_heads, head_dim, page_size, _dtype_code(dtype), float(sm_scale))


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None or t.numel() == 0 else t.data_ptr()


_I32 = torch.int32


def paged_kv(part) -> PagedKV:
    """Marshal an object with k_pool, v_pool, page_indptr, page_indices, seq_lens tensors."""
    kp, vp, indptr, indices, lens = part.k_pool, part.v_pool, part.page_indptr, part.page_indices, part.seq_lens
    assert (kp.is_contiguous() and vp.is_contiguous() and indptr.is_contiguous() and indices.is_contiguous() and lens.is_contiguous() and
            indptr.dtype is _I32 and indices.dtype is _I32 and lens.dtype is _I32)
    pages = kp.shape[0]
    return PagedKV(kp.data_ptr() if pages else _ptr(kp), vp.data_ptr() if pages else _ptr(vp), pages,
                   indptr.data_ptr(), _ptr(indices), lens.data_ptr())


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is not None:
        return stream.cuda_stream
    try:                        # torch.cuda.current_stream() without the wrapper object: 3 us less per call, but not a documented function
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    except AttributeError:
        return torch.cuda.current_stream().cuda_stream


def _current_device() -> int:
    try:
        return torch._C._cuda_getDevice()
    except AttributeError:
        return torch.cuda.current_device()


def spd_workspace_size(shape: Shape) -> int:
    n = C.c_size_t(0)
    _check(lib().spd_workspace_size(C.byref(shape), C.byref(n)), "spd_workspace_size")
    return int(n.value)


def alloc_workspace(shape: Shape, device="cuda") -> torch.Tensor:
    """A zeroed workspace tensor of the size the library asks for."""
    return torch.zeros(spd_workspace_size(shape), dtype=torch.uint8, device=device)


def alloc_partial(shape: Shape, device="cuda") -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    B, H, D = shape.batch, shape.num_q_heads, shape.head_dim
    return (torch.empty((B, H, D), dtype=torch.float32, device=device),
            torch.empty((B, H), dtype=torch.float32, device=device),
            torch.empty((B, H), dtype=torch.float32, device=device))


def spd_partial_attn(shape, q, priv, out, ws, stream=None, plan=None) -> None:
    """plan=None calls spd_partial_attn; SPD_PLAN_* calls spd_partial_attn_planned with that mode."""
    kv = paged_kv(priv)
    part = Partial(out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr())
    if plan is None:
        _check(lib().spd_partial_attn(C.byref(shape), q.data_ptr(), C.byref(kv), part, ws.data_ptr(), ws.numel(),
                                      _stream_ptr(stream)), "spd_partial_attn")
    else:
        _check(lib().spd_partial_attn_planned(C.byref(shape), q.data_ptr(), C.byref(kv), part, int(plan), ws.data_ptr(),
                                              ws.numel(), _stream_ptr(stream)), "spd_partial_attn_planned")


def spd_service_attn_merge(shape, q, pub, partial_in, out, ws, stream=None, plan=None) -> None:
    kv = paged_kv(pub)
    part = Partial(partial_in[0].data_ptr(), partial_in[1].data_ptr(), partial_in[2].data_ptr())
    if plan is None:
        _check(lib().spd_service_attn_merge(C.byref(shape), q.data_ptr(), C.byref(kv), part, out.data_ptr(),
                                            _dtype_code(out.dtype), ws.data_ptr(), ws.numel(), _stream_ptr(stream)),
               "spd_service_attn_merge")
    else:
        _check(lib().spd_service_attn_merge_planned(C.byref(shape), q.data_ptr(), C.byref(kv), part, out.data_ptr(),
                                                    _dtype_code(out.dtype), int(plan), ws.data_ptr(), ws.numel(),
                                                    _stream_ptr(stream)), "spd_service_attn_merge_planned")


def spd_decode_step(shape, q, priv, pub, out, ws, fused=True, stream=None, plan=None) -> None:
    a, b = paged_kv(priv), paged_kv(pub)
    if plan is None:
        _check(lib().spd_decode_step(C.byref(shape), q.data_ptr(), C.byref(a), C.byref(b), out.data_ptr(),
                                     _dtype_code(out.dtype), 1 if fused else 0, ws.data_ptr(), ws.numel(),
                                     _stream_ptr(stream)), "spd_decode_step")
    else:
        _check(lib().spd_decode_step_planned(C.byref(shape), q.data_ptr(), C.byref(a), C.byref(b), out.data_ptr(),
                                             _dtype_code(out.dtype), 1 if fused else 0, int(plan), ws.data_ptr(),
                                             ws.numel(), _stream_ptr(stream)), "spd_decode_step_planned")


def spd_step_blob_layout(shape, priv_pages_listed: int, pub_pages_listed: int, out_dtype) -> StepBlob:
    lay = StepBlob()
    _check(lib().spd_step_blob_layout(C.byref(shape), priv_pages_listed, pub_pages_listed,
                                      _dtype_code(out_dtype), C.byref(lay)), "spd_step_blob_layout")
    return lay


def spd_decode_step_host(shape, layout, host_blob, device_blob, priv_pools, pub_pools, out_dtype, ws,
                         stream=None) -> Tuple[int, int]:
    """host_blob: pinned uint8 host tensor laid out per `layout`; device_blob: uint8 device tensor of
    layout.total_bytes; *_pools: (k_pool, v_pool) device tensors.  Waits for the stream; the output is
    then at host_blob[layout.out:].  Returns (device status, first flagged user or -1)."""
    def kv(pools):
        return PagedKV(_ptr(pools[0]), _ptr(pools[1]), int(pools[0].shape[0]), None, None, None)
    a, b = kv(priv_pools), kv(pub_pools)
    bad = C.c_int32(-1)
    code = lib().spd_decode_step_host(C.byref(shape), C.byref(layout), host_blob.data_ptr(), device_blob.data_ptr(),
                                      C.byref(a), C.byref(b), _dtype_code(out_dtype), C.byref(bad), ws.data_ptr(),
                                      ws.numel(), _stream_ptr(stream))
    if code not in _DEVICE_CODES:
        raise SpdError(code, "spd_decode_step_host")
    return int(code), int(bad.value)


class HostStep:
    """spd_decode_step_host with its arguments marshalled once: for a serving loop that reuses the same
    buffers every step and only rewrites the host blob.  Calling the object runs one step."""

    def __init__(self, shape, layout, host_blob, device_blob, priv_pools, pub_pools, out_dtype, ws, stream=None):
        self._keep = (shape, layout, host_blob, device_blob, priv_pools, pub_pools, ws)   # keep the memory alive
        self._a = PagedKV(_ptr(priv_pools[0]), _ptr(priv_pools[1]), int(priv_pools[0].shape[0]), None, None, None)
        self._b = PagedKV(_ptr(pub_pools[0]), _ptr(pub_pools[1]), int(pub_pools[0].shape[0]), None, None, None)
        self._bad = C.c_int32(-1)
        self._fn = lib().spd_decode_step_host
        self._args = (C.byref(shape), C.byref(layout), C.c_void_p(host_blob.data_ptr()), C.c_void_p(device_blob.data_ptr()),
                      C.byref(self._a), C.byref(self._b), _dtype_code(out_dtype), C.byref(self._bad),
                      C.c_void_p(ws.data_ptr()), C.c_size_t(ws.numel()), C.c_void_p(_stream_ptr(stream)))

    def __call__(self) -> Tuple[int, int]:
        code = self._fn(*self._args)
        if code not in _DEVICE_CODES:
            raise SpdError(code, "spd_decode_step_host")
        return int(code), int(self._bad.value)


def fill_step_blob(layout, host_blob, q, priv, pub) -> None:
    """Copy q and the two partitions' tables (any device) into a host blob at the layout's offsets."""
    def put(off, t):
        src = t.detach().cpu().contiguous().view(torch.uint8).reshape(-1)
        host_blob[off:off + src.numel()] = src
    put(layout.q, q)
    for part, (a, b, c) in ((priv, (layout.priv_indptr, layout.priv_lens, layout.priv_indices)),
                            (pub, (layout.pub_indptr, layout.pub_lens, layout.pub_indices))):
        put(a, part.page_indptr)
        put(b, part.seq_lens)
        put(c, part.page_indices)


def spd_query_device_status(ws, stream=None) -> Tuple[int, int]:
    """Waits for the stream; returns (status code, first flagged user or -1) and clears the flag."""
    bad = C.c_int32(-1)
    code = lib().spd_query_device_status(ws.data_ptr(), _stream_ptr(stream), C.byref(bad))
    return int(code), int(bad.value)


def spd_kernel_launch_count() -> int:
    return int(lib().spd_kernel_launch_count())


def spd_profile_begin(max_calls: int) -> None:
    _check(lib().spd_profile_begin(int(max_calls)), "spd_profile_begin")


def spd_profile_end() -> dict:
    """Returns {'calls', 'kernel_ms'}: calls recorded and their summed kernel time."""
    n, a = C.c_int32(0), C.c_double(0)
    _check(lib().spd_profile_end(C.byref(n), C.byref(a)), "spd_profile_end")
    return dict(calls=int(n.value), kernel_ms=a.value)


STATIC_WS_BYTES = 16 << 20


def spd_decode_step_static(shape, q, priv, pub, out, wait_and_check=True, stream=None) -> Tuple[int, int]:
    """The fused decode step with the workspace held inside the library (nothing is allocated).

    For callers that cannot allocate device memory; the shape must need at most STATIC_WS_BYTES of
    workspace.  Returns (status, first flagged user or -1); status is SPD_OK when not waiting.
    Raises SpdError for host-side rejections such as a shape beyond the limit."""
    a, b = paged_kv(priv), paged_kv(pub)
    bad = C.c_int32(-1)
    code = lib().spd_decode_step_static(C.byref(shape), q.data_ptr(), C.byref(a), C.byref(b), out.data_ptr(),
                                        _dtype_code(out.dtype), 1 if wait_and_check else 0, C.byref(bad),
                                        _stream_ptr(stream))
    if code not in _DEVICE_CODES:
        raise SpdError(code, "spd_decode_step_static")
    return int(code), int(bad.value)


def spd_append_kv(shape, k_new, v_new, part, ws, stream=None) -> None:
    """Append one token per user to the partition `part` (its pools and seq_lens are updated in place)."""
    assert k_new.is_contiguous() and v_new.is_contiguous()
    _check(lib().spd_append_kv(C.byref(shape), k_new.data_ptr(), v_new.data_ptr(), part.k_pool.data_ptr(),
                               part.v_pool.data_ptr(), int(part.k_pool.shape[0]), part.page_indptr.data_ptr(),
                               _ptr(part.page_indices), part.seq_lens.data_ptr(), ws.data_ptr(), ws.numel(),
                               _stream_ptr(stream)), "spd_append_kv")


def spd_decode_step_append(shape, q, k_new, v_new, priv, pub, out, ws, plan=SPD_PLAN_PER_CALL, stream=None) -> None:
    """The append of the new token's rows to `pub` (pools and seq_lens updated in place) and the fused decode step
    over the grown cache, in one launch."""
    assert k_new.is_contiguous() and v_new.is_contiguous()
    a, b = paged_kv(priv), paged_kv(pub)
    _check(lib().spd_decode_step_append(C.byref(shape), q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), C.byref(a),
                                        C.byref(b), out.data_ptr(), _dtype_code(out.dtype), int(plan), ws.data_ptr(),
                                        ws.numel(), _stream_ptr(stream)), "spd_decode_step_append")


def spd_service_attn_merge_append(shape, q, k_new, v_new, pub, partial_in, out, ws, plan=SPD_PLAN_PER_CALL, stream=None) -> None:
    """The service call with the append at its head: `pub` grows by the new token (pools and seq_lens updated in
    place), its partial is merged with `partial_in` and the attention output written, in one launch."""
    assert k_new.is_contiguous() and v_new.is_contiguous()
    kv = paged_kv(pub)
    part = Partial(partial_in[0].data_ptr(), partial_in[1].data_ptr(), partial_in[2].data_ptr())
    _check(lib().spd_service_attn_merge_append(C.byref(shape), q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), C.byref(kv),
                                               part, out.data_ptr(), _dtype_code(out.dtype), int(plan), ws.data_ptr(),
                                               ws.numel(), _stream_ptr(stream)), "spd_service_attn_merge_append")


def spd_token_step(shape, layers, ws, stream=None, same_lengths=False) -> None:
    """layers: a sequence of (q, k_new, v_new, priv, pub, out) per layer; appends to each pub and runs each decode step.
    same_lengths: every layer's lengths equal layer 0's, so its plan is derived once and reused."""
    arr = (Layer * len(layers))()
    for i, (q, k_new, v_new, priv, pub, out) in enumerate(layers):
        assert q.is_contiguous() and k_new.is_contiguous() and v_new.is_contiguous() and out.is_contiguous()
        arr[i] = Layer(q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), paged_kv(priv), paged_kv(pub), out.data_ptr())
    _check(lib().spd_token_step(C.byref(shape), len(layers), arr, _dtype_code(layers[0][5].dtype),
                                1 if same_lengths else 0, ws.data_ptr(), ws.numel(), _stream_ptr(stream)), "spd_token_step")


def _watch(tok_lo, tok_hi, out) -> Watch:
    assert tok_lo.dtype == torch.int32 and tok_hi.dtype == torch.int32 and out.dtype == torch.float32
    return Watch(tok_lo.data_ptr(), tok_hi.data_ptr(), out.data_ptr())


def spd_partial_attn_watch(shape, q, priv, out, tok_lo, tok_hi, watch_out, ws, stream=None) -> None:
    kv, w = paged_kv(priv), _watch(tok_lo, tok_hi, watch_out)
    part = Partial(out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr())
    _check(lib().spd_partial_attn_watch(C.byref(shape), q.data_ptr(), C.byref(kv), part, C.byref(w), ws.data_ptr(),
                                        ws.numel(), _stream_ptr(stream)), "spd_partial_attn_watch")


def spd_decode_step_watch(shape, q, priv, pub, out, tok_lo, tok_hi, watch_out, ws, stream=None) -> None:
    a, b, w = paged_kv(priv), paged_kv(pub), _watch(tok_lo, tok_hi, watch_out)
    _check(lib().spd_decode_step_watch(C.byref(shape), q.data_ptr(), C.byref(a), C.byref(b), out.data_ptr(),
                                       _dtype_code(out.dtype), C.byref(w), ws.data_ptr(), ws.numel(),
                                       _stream_ptr(stream)), "spd_decode_step_watch")


def spd_watch_alarm(mass, threshold: float, head_mask=None):
    """mass: float32 HOST tensor [batch, heads] from a *_watch call; head_mask: optional bool/uint8 [heads].
    Returns (alarm int32 [batch], score float32 [batch]): score = mean watched mass over the selected heads,
    alarm = 1 where it is below the threshold."""
    assert mass.device.type == "cpu" and mass.dtype == torch.float32 and mass.is_contiguous() and mass.dim() == 2
    B, H = mass.shape
    alarm = torch.zeros(B, dtype=torch.int32)
    score = torch.zeros(B, dtype=torch.float32)
    hm = None if head_mask is None else head_mask.to(torch.uint8).contiguous()
    _check(lib().spd_watch_alarm(mass.data_ptr(), B, H, None if hm is None else hm.data_ptr(), float(threshold),
                                 alarm.data_ptr(), score.data_ptr()), "spd_watch_alarm")
    return alarm, score


def spd_set_bf16_math(path: int) -> None:
    """0 = tensor cores (default), 1 = FMA pipes (comparison arm); process-wide."""
    _check(lib().spd_set_bf16_math(int(path)), "spd_set_bf16_math")


def spd_set_split(min_tiles_per_share: int = 0, uniform_shares: bool = False) -> None:
    """How the tile stream is cut from now on, process-wide: fewest tiles per share (0 = default) and whether
    every CTA weighs the same (the measured rates are ignored; results become repeatable bit for bit)."""
    _check(lib().spd_set_split(int(min_tiles_per_share), 1 if uniform_shares else 0), "spd_set_split")


def spd_set_programmatic_launch(on: bool) -> None:
    _check(lib().spd_set_programmatic_launch(1 if on else 0), "spd_set_programmatic_launch")


def spd_debug_read_plan(ws, which: int = 2, stream=None, capacity: int = 256 * 16 + 1):
    """(tiles, shares, bnd) of the last derived plan of kind `which` (0 private only, 1 public only, 2 both)."""
    T, A = C.c_int32(0), C.c_int32(0)
    bnd = (C.c_int32 * capacity)()
    _check(lib().spd_debug_read_plan(ws.data_ptr(), int(which), _stream_ptr(stream), C.byref(T), C.byref(A), bnd, capacity),
           "spd_debug_read_plan")
    n = min(capacity, A.value + 1)
    return int(T.value), int(A.value), [int(bnd[i]) for i in range(n)]


def spd_debug_sm_moves(ws, stream=None) -> Tuple[int, int]:
    """(launches that could compare, CTAs that ran on another SM than the same CTA index one launch earlier)."""
    a, b = C.c_int64(0), C.c_int64(0)
    _check(lib().spd_debug_sm_moves(ws.data_ptr(), _stream_ptr(stream), C.byref(a), C.byref(b)), "spd_debug_sm_moves")
    return int(a.value), int(b.value)


def spd_set_prefill_rows(rows: int) -> None:
    """Query rows per prefill CTA: 0 = chosen per call from the mean prompt length (default), 128 or 256; process-wide."""
    _check(lib().spd_set_prefill_rows(int(rows)), "spd_set_prefill_rows")


def spd_merge_partials(shape, parts, out, stream=None) -> None:
    """parts: a sequence of (o, m, l) tensor triples; writes the merged, normalised output."""
    arr = (Partial * len(parts))(*[Partial(o.data_ptr(), m.data_ptr(), l.data_ptr()) for o, m, l in parts])
    _check(lib().spd_merge_partials(C.byref(shape), len(parts), arr, out.data_ptr(), _dtype_code(out.dtype),
                                    _stream_ptr(stream)), "spd_merge_partials")


def spd_prefill_attn(shape, q, k, v, tok_indptr, part, out, ws, stream=None) -> None:
    """Causal attention over the prompts (q [T,Hq,D], k, v [T,Hkv,D], tok_indptr int32 [B+1]) into `out`
    [T,Hq,D]; the prompts' K/V rows go into the partition `part` (pools and seq_lens updated in place)."""
    for t in (q, k, v, out):
        assert t.is_contiguous()
    assert tok_indptr.dtype == torch.int32
    _check(lib().spd_prefill_attn(C.byref(shape), int(q.shape[0]), _ptr(q), _ptr(k), _ptr(v), tok_indptr.data_ptr(),
                                  part.k_pool.data_ptr(), part.v_pool.data_ptr(), int(part.k_pool.shape[0]),
                                  part.page_indptr.data_ptr(), _ptr(part.page_indices), part.seq_lens.data_ptr(),
                                  _ptr(out), _dtype_code(out.dtype), ws.data_ptr(), ws.numel(), _stream_ptr(stream)),
           "spd_prefill_attn")


def make_score(logit_cap: float = 0.0, window: int = 0, alibi_slopes: Optional[torch.Tensor] = None) -> Score:
    """Score options of the *_scored calls; alibi_slopes: float32 [num_q_heads] on the device."""
    if not -2**31 <= window < 2**31:
        raise ValueError("the window is a 32-bit number")
    sc = Score(float(logit_cap), int(window), None)
    if alibi_slopes is not None:
        if alibi_slopes.dtype is not torch.float32 or not alibi_slopes.is_contiguous() or not alibi_slopes.is_cuda:
            raise ValueError(f"slopes are contiguous float32 on the device, got {alibi_slopes.dtype} on {alibi_slopes.device}")
        sc.alibi_slopes = alibi_slopes.data_ptr()
        sc._keep = alibi_slopes
    return sc


def make_rope(inv_freq: torch.Tensor, interleaved: bool = False, sections=None, scale: float = 1.0) -> Rope:
    """Rotation of spd_append_kv_rope; inv_freq: float32 [rotary_dim / 2] on the device; sections: pairs per position axis."""
    if inv_freq.dtype is not torch.float32 or not inv_freq.is_contiguous() or not inv_freq.is_cuda or inv_freq.dim() != 1:
        raise ValueError(f"inv_freq is contiguous float32 [rotary_dim / 2] on the device, got {inv_freq.dtype} {list(inv_freq.shape)} on {inv_freq.device}")
    rope = Rope(2 * inv_freq.numel(), 1 if interleaved else 0, len(sections) if sections else 1, _Sections(*(sections or ())),
                float(scale), inv_freq.data_ptr())
    rope._keep = inv_freq
    return rope


_TORCH_DTYPES = {SPD_F32: torch.float32, SPD_BF16: torch.bfloat16}

# Checks of the tensors whose addresses a call hands over.  `dev` is the device that the call runs on; an address on another device or
# on the host, or a tensor smaller than the kernels read or write, would fault there.


def _elsewhere(t: torch.Tensor) -> ValueError:
    return ValueError(f"expected a tensor on the current CUDA device, got one on {t.device}")


def _here(t: torch.Tensor) -> int:
    """The tensors of a call live on the current device, whose stream and context the call uses; its index."""
    dev = t.get_device()
    if dev < 0 or dev != _current_device():
        raise _elsewhere(t)
    return dev


def _slopes(shape, score, dev) -> None:
    keep = getattr(score, "_keep", None)
    if keep is None:
        return
    if keep.numel() != shape.num_q_heads:
        raise ValueError(f"one slope per query head: expected {shape.num_q_heads}, got {keep.numel()}")
    if keep.get_device() != dev:
        raise _elsewhere(keep)


def _rows(t: torch.Tensor, heads: int, d: int, n: int, dtype, dev=None):
    """(pointer, token stride in elements) of [n, heads, d] rows that may be part of a wider row per token."""
    if t.dtype is not dtype or t.shape != (n, heads, d):
        raise ValueError(f"expected {dtype} [{n}, {heads}, {d}], got {t.dtype} {list(t.shape)}")
    if n == 0:
        return None, 0
    if t.get_device() != dev:
        raise _elsewhere(t)
    if t.is_contiguous():
        return t.data_ptr(), 0
    s0, s1, s2 = t.stride()
    if s2 != 1 or (heads > 1 and s1 != d):
        raise ValueError("a token's heads must be packed")
    if n > 1 and s0 < heads * d:            # an expanded tensor's 0 would read as packed
        raise ValueError("tokens must not overlap")
    return t.data_ptr(), s0 if n > 1 else 0


def _i32(t: Optional[torch.Tensor], *size, dev=None) -> Optional[int]:
    """Pointer of a contiguous int32 tensor of the given shape, or None."""
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.shape != size or not t.is_contiguous():
        raise ValueError(f"expected contiguous int32 {list(size)}, got {t.dtype} {list(t.shape)}")
    if t.get_device() != dev:
        raise _elsewhere(t)
    return t.data_ptr()


def _packed(t: Optional[torch.Tensor], numel: int, dtype=None, dev=None) -> Optional[int]:
    """Pointer of a contiguous tensor of `numel` elements, or None."""
    if t is None:
        return None
    if t.numel() != numel or not t.is_contiguous() or (dtype is not None and t.dtype is not dtype):
        raise ValueError(f"expected a contiguous tensor of {numel} elements, got {t.dtype} {list(t.shape)}")
    if t.get_device() != dev:
        raise _elsewhere(t)
    return t.data_ptr() if numel else None


def _workspace(ws: torch.Tensor, dev):
    """(pointer, bytes) of a workspace."""
    if ws.get_device() != dev or ws.dtype is not torch.uint8 or not ws.is_contiguous():
        raise ValueError(f"a workspace is a contiguous uint8 tensor on the current CUDA device, got {ws.dtype} on {ws.device}")
    return ws.data_ptr(), ws.numel()


def _partition(part, B, page, dtype, dev):
    """The fields of PagedKV, in order: pools of pages of `page` elements, a table and a length per user."""
    kp, vp, indptr, indices, lens = part.k_pool, part.v_pool, part.page_indptr, part.page_indices, part.seq_lens
    pages = kp.shape[0]
    if not (kp.dtype is dtype and vp.dtype is dtype and kp.numel() == pages * page == vp.numel() and kp.is_contiguous() and vp.is_contiguous()):
        raise ValueError(f"expected contiguous {dtype} pools of {pages} pages of {page} elements (KV heads x page size x head_dim), got "
                         f"{kp.dtype} {list(kp.shape)} and {vp.dtype} {list(vp.shape)}")
    if not (indptr.dtype is _I32 and indices.dtype is _I32 and lens.dtype is _I32 and indptr.numel() == B + 1 and lens.numel() == B and
            indptr.is_contiguous() and indices.is_contiguous() and lens.is_contiguous()):
        raise ValueError(f"expected contiguous int32 page_indptr [{B + 1}], page_indices and seq_lens [{B}], got {indptr.dtype} "
                         f"{list(indptr.shape)}, {indices.dtype} and {lens.dtype} {list(lens.shape)}")
    if not (kp.get_device() == dev == vp.get_device() and indptr.get_device() == dev == indices.get_device() and lens.get_device() == dev):
        raise _elsewhere(next(t for t in (kp, vp, indptr, indices, lens) if t.get_device() != dev))
    return kp.data_ptr(), vp.data_ptr(), pages, indptr.data_ptr(), indices.data_ptr(), lens.data_ptr()      # an empty tensor's is 0


def _query(shape, q):
    """One packed query row per user and head.  The device of the call, and what its partitions are held against."""
    dev, B, d, dtype = _here(q), shape.batch, shape.head_dim, _TORCH_DTYPES[shape.dtype]
    _packed(q, B * shape.num_q_heads * d, dtype, dev)
    return dev, (B, shape.num_kv_heads * shape.page_size * d, dtype, dev)


def _partial(shape, part, dev) -> Partial:
    rows = shape.batch * shape.num_q_heads
    return Partial(_packed(part[0], rows * shape.head_dim, torch.float32, dev), _packed(part[1], rows, torch.float32, dev),
                   _packed(part[2], rows, torch.float32, dev))


def spd_partial_attn_scored(shape, score, q, priv, pub_lens, out, ws, plan=SPD_PLAN_PER_CALL, stream=None) -> None:
    """spd_partial_attn with score options; pub_lens: int32 [batch], tokens in the public partition."""
    dev, fit = _query(shape, q)
    _slopes(shape, score, dev)
    kv, part = PagedKV(*_partition(priv, *fit)), _partial(shape, out, dev)
    _check(lib().spd_partial_attn_scored(shape, score, q.data_ptr(), kv, _i32(pub_lens, shape.batch, dev=dev), part, plan, *_workspace(ws, dev),
                                         _stream_ptr(stream)), "spd_partial_attn_scored")


def spd_service_attn_merge_scored(shape, score, q, pub, priv_lens, partial_in, out, ws, plan=SPD_PLAN_PER_CALL, stream=None) -> None:
    """spd_service_attn_merge with score options; priv_lens: int32 [batch], tokens in the private partition."""
    dev, fit = _query(shape, q)
    _slopes(shape, score, dev)
    kv, part = PagedKV(*_partition(pub, *fit)), _partial(shape, partial_in, dev)
    _check(lib().spd_service_attn_merge_scored(shape, score, q.data_ptr(), kv, _i32(priv_lens, shape.batch, dev=dev), part,
                                               _packed(out, q.numel(), dev=dev), _dtype_code(out.dtype), plan, *_workspace(ws, dev),
                                               _stream_ptr(stream)), "spd_service_attn_merge_scored")


def spd_decode_step_scored(shape, score, q, priv, pub, out, ws, plan=SPD_PLAN_PER_CALL, stream=None) -> None:
    """The fused decode step with score options (make_score) over both partitions."""
    dev, fit = _query(shape, q)
    _slopes(shape, score, dev)
    a, b = PagedKV(*_partition(priv, *fit)), PagedKV(*_partition(pub, *fit))
    _check(lib().spd_decode_step_scored(shape, score, q.data_ptr(), a, b, _packed(out, q.numel(), dev=dev), _dtype_code(out.dtype), plan,
                                        *_workspace(ws, dev), _stream_ptr(stream)), "spd_decode_step_scored")


def spd_prefill_attn_scored(shape, score, q, k, v, tok_indptr, out, ws, prefix_lens=None, doc_start=None, stream=None) -> None:
    """Prompt attention with score options and interval masks: q [T,Hq,D], k, v [T,Hkv,D] (rows may be parts of a wider row per
    token), tok_indptr int32 [B+1], prefix_lens int32 [B], doc_start int32 [T], out [T,Hq,D] packed."""
    dev = _here(q)
    _slopes(shape, score, dev)
    T, B, hq, hkv, d, dtype = q.shape[0], shape.batch, shape.num_q_heads, shape.num_kv_heads, shape.head_dim, _TORCH_DTYPES[shape.dtype]
    qp, qs = _rows(q, hq, d, T, dtype, dev)
    kp, ks = _rows(k, hkv, d, T, dtype, dev)
    vp, vs = _rows(v, hkv, d, T, dtype, dev)
    _check(lib().spd_prefill_attn_scored(shape, score, T, Tokens(qp, kp, vp, qs, ks, vs), _i32(tok_indptr, B + 1, dev=dev),
                                         _i32(prefix_lens, B, dev=dev), _i32(doc_start, T, dev=dev), _packed(out, T * hq * d, dev=dev),
                                         _dtype_code(out.dtype), *_workspace(ws, dev), _stream_ptr(stream)), "spd_prefill_attn_scored")


def spd_append_kv_rope(shape, rope, q, k, v, part, ws, q_out=None, k_out=None, tok_indptr=None, positions=None, pos_base=None,
                       new_lens="in place", stream=None) -> None:
    """Rotate the new tokens' q and k rows (into q_out, k_out) and append k and v to the partition `part`.

    rope: make_rope(...) or None (no rotation; q and q_out are not used).  tok_indptr int32 [B+1]: tokens per user; None: one
    token per user.  positions int32 [axes, T] or [T]; pos_base int32 [B].  new_lens: an int32 [B] tensor, None, or by default
    part.seq_lens itself."""
    dev = _here(k)
    T, B, hq, hkv, d, dtype = k.shape[0], shape.batch, shape.num_q_heads, shape.num_kv_heads, shape.head_dim, _TORCH_DTYPES[shape.dtype]
    kp, ks = _rows(k, hkv, d, T, dtype, dev)
    vp, vs = _rows(v, hkv, d, T, dtype, dev)
    qp, qs = _rows(q, hq, d, T, dtype, dev) if rope is not None else (None, 0)
    if rope is not None:
        keep = getattr(rope, "_keep", None)
        if keep is not None and keep.get_device() != dev:
            raise _elsewhere(keep)
    if positions is not None:
        if rope is None:
            raise ValueError("positions are for a rotation")
        positions = _i32(positions, T, dev=dev) if positions.dim() == 1 and rope.num_axes == 1 else _i32(positions, rope.num_axes, T, dev=dev)
    pool_k, pool_v, pages, indptr, indices, lens = _partition(part, B, hkv * shape.page_size * d, dtype, dev)
    _check(lib().spd_append_kv_rope(shape, rope, T, Tokens(qp, kp, vp, qs, ks, vs), _i32(tok_indptr, B + 1, dev=dev), positions,
                                    _i32(pos_base, B, dev=dev), _packed(q_out, T * hq * d, dtype, dev), _packed(k_out, T * hkv * d, dtype, dev),
                                    pool_k, pool_v, pages, indptr, indices, lens,
                                    lens if isinstance(new_lens, str) else _i32(new_lens, B, dev=dev), *_workspace(ws, dev),
                                    _stream_ptr(stream)), "spd_append_kv_rope")


def spd_drafted_workspace_size(shape: Shape) -> int:
    n = C.c_size_t(0)
    _check(lib().spd_drafted_workspace_size(C.byref(shape), C.byref(n)), "spd_drafted_workspace_size")
    return int(n.value)


def alloc_drafted_workspace(shape: Shape, device="cuda") -> torch.Tensor:
    """A zeroed workspace for the *_drafted calls, and for every other call of the shape."""
    return torch.zeros(spd_drafted_workspace_size(shape), dtype=torch.uint8, device=device)


def _ints(t, n, dev):
    """Pointer of n int32 numbers one after the other on the call's device, or None.  (_i32 without the shape: half its time.)"""
    if t is None:
        return None
    if t.dtype is _I32 and t.numel() == n and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    if t.dtype is _I32 and t.numel() == n and t.is_contiguous():
        raise _elsewhere(t)
    raise ValueError(f"expected contiguous int32 of {n} elements, got {t.dtype} {list(t.shape)}")


def _drafted(shape, score, q, tok_indptr, parents, sinks):
    """What the *_drafted calls have in common: the drafts, the rows' count, the device, and what partitions are held against."""
    dev, T, B, hq, d, dtype = _here(q), q.shape[0], shape.batch, shape.num_q_heads, shape.head_dim, _TORCH_DTYPES[shape.dtype]
    if q.dtype is not dtype or q.numel() != T * hq * d or not q.is_contiguous():
        raise ValueError(f"expected contiguous {dtype} [tokens, {hq}, {d}], got {q.dtype} {list(q.shape)}")
    if not 0 <= sinks < 2**31:
        raise ValueError("the number of sinks is a 32-bit number, not negative")
    if tok_indptr is None and T != B:
        raise ValueError(f"{T} tokens of {B} users need a tok_indptr")
    if score.alibi_slopes is not None:
        _slopes(shape, score, dev)
    return Drafts(T, _ints(tok_indptr, B + 1, dev), _ints(parents, T, dev), sinks), T, dev, (B, shape.num_kv_heads * shape.page_size * d, dtype, dev)


def _drafted_partial(shape, part, T, dev) -> Partial:
    rows = T * shape.num_q_heads
    return Partial(_packed(part[0], rows * shape.head_dim, torch.float32, dev), _packed(part[1], rows, torch.float32, dev),
                   _packed(part[2], rows, torch.float32, dev))


def spd_decode_step_drafted(shape, score, q, priv, pub, out, ws, tok_indptr=None, parents=None, sinks=0, stream=None) -> None:
    """One decode step for several tokens per user, the last ones of the public partition: q, out [T,Hq,D]; tok_indptr int32 [B+1] (None: one
    token per user); parents int32 [T], a tree (None: runs); sinks: first tokens that stay visible behind the window."""
    drafts, T, dev, fit = _drafted(shape, score, q, tok_indptr, parents, sinks)
    a, b = PagedKV(*_partition(priv, *fit)), PagedKV(*_partition(pub, *fit))
    _check(lib().spd_decode_step_drafted(shape, score, drafts, _ptr(q), a, b, _packed(out, q.numel(), dev=dev), _dtype_code(out.dtype),
                                         *_workspace(ws, dev), _stream_ptr(stream)), "spd_decode_step_drafted")


def spd_partial_attn_drafted(shape, score, q, priv, pub_lens, out, ws, tok_indptr=None, parents=None, sinks=0, stream=None) -> None:
    """The private half of spd_decode_step_drafted: out = (o [T,Hq,D], m [T,Hq], l [T,Hq]); pub_lens int32 [B] counts the drafted tokens."""
    drafts, T, dev, fit = _drafted(shape, score, q, tok_indptr, parents, sinks)
    kv, part = PagedKV(*_partition(priv, *fit)), _drafted_partial(shape, out, T, dev)
    _check(lib().spd_partial_attn_drafted(shape, score, drafts, _ptr(q), kv, _ints(pub_lens, shape.batch, dev), part, *_workspace(ws, dev),
                                          _stream_ptr(stream)), "spd_partial_attn_drafted")


def spd_service_attn_merge_drafted(shape, score, q, pub, priv_lens, partial_in, out, ws, tok_indptr=None, parents=None, sinks=0, stream=None) -> None:
    """The public half of spd_decode_step_drafted, merged with the private partial and normalised; priv_lens int32 [B]."""
    drafts, T, dev, fit = _drafted(shape, score, q, tok_indptr, parents, sinks)
    kv, part = PagedKV(*_partition(pub, *fit)), _drafted_partial(shape, partial_in, T, dev)
    _check(lib().spd_service_attn_merge_drafted(shape, score, drafts, _ptr(q), kv, _ints(priv_lens, shape.batch, dev), part,
                                                _packed(out, q.numel(), dev=dev), _dtype_code(out.dtype), *_workspace(ws, dev),
                                                _stream_ptr(stream)), "spd_service_attn_merge_drafted")


def _layout(shape):
    """What the rows of a pool's pages go by."""
    return shape.num_kv_heads, shape.page_size, shape.head_dim, shape.dtype


class Pools:
    """Pools that share their pages' tables, K and V of any number of layers, as the calls take them; it keeps them alive."""

    def __init__(self, shape, pools):
        pools = list(pools)
        self.dev = _here(pools[0]) if pools else -1
        self.pages, self.layout = (pools[0].shape[0] if pools else 0), _layout(shape)
        page, dtype = shape.num_kv_heads * shape.page_size * shape.head_dim, _TORCH_DTYPES[shape.dtype]
        for t in pools:
            if t.dtype is not dtype or t.shape[0] != self.pages or t.numel() != self.pages * page or not t.is_contiguous():
                raise ValueError(f"expected contiguous {dtype} pools of {self.pages} pages of {page} elements (KV heads x page size x "
                                 f"head_dim), got {t.dtype} {list(t.shape)}")
            if t.get_device() != self.dev:
                raise _elsewhere(t)
        self.count, self.array, self._keep = len(pools), (C.c_void_p * max(1, len(pools)))(*[t.data_ptr() for t in pools]), pools


def make_pools(shape, pools) -> Pools:
    """A handle for spd_keep_drafted and spd_pages_copy, for a program that keeps its pools: the list is looked over once."""
    return Pools(shape, pools)


def _pools(shape, pools, dev) -> Pools:
    if not isinstance(pools, Pools):
        pools = Pools(shape, pools)
    elif pools.layout != _layout(shape):
        raise ValueError("the pools were made for another shape")
    if pools.count and pools.dev != dev:
        raise _elsewhere(pools._keep[0])
    return pools


def spd_keep_drafted(shape, pools, part, tok_indptr, last, ws, parents=None, new_lens="in place", kept=None, total_tokens=None, stream=None) -> None:
    """Keep token last[u] (int32 [B], -1 = none) of each user's drafted tokens and those that it comes after: their rows move to the front in
    all `pools` (make_pools, or a list of tensors), whose tables and lengths `part` has; tok_indptr int32 [B+1] or None (one token per user);
    parents int32 [T] or None (runs); new_lens: an int32 [B] tensor, None, or by default part.seq_lens itself; kept int32 [T] or None;
    total_tokens: T, where neither parents nor kept tells it."""
    dev, B = _here(last), shape.batch
    T = B if tok_indptr is None else next((t.numel() for t in (parents, kept) if t is not None), total_tokens)
    if T is None:
        raise ValueError("total_tokens is needed")
    pools = _pools(shape, pools, dev)
    lens, indices = _ints(part.seq_lens, B, dev), part.page_indices
    new_lens = lens if isinstance(new_lens, str) else _ints(new_lens, B, dev)
    _check(lib().spd_keep_drafted(shape, T, _ints(tok_indptr, B + 1, dev), _ints(parents, T, dev), _ints(last, B, dev), pools.count, pools.array, pools.pages,
                                  _ints(part.page_indptr, B + 1, dev), _ints(indices, indices.numel(), dev), lens, new_lens, _ints(kept, T, dev),
                                  *_workspace(ws, dev), _stream_ptr(stream)), "spd_keep_drafted")


def spd_pages_workspace_size(shape: Shape, num_pages: int) -> int:
    n = C.c_size_t(0)
    _check(lib().spd_pages_workspace_size(shape, num_pages, C.byref(n)), "spd_pages_workspace_size")
    return int(n.value)


def alloc_pages_workspace(shape: Shape, num_pages: int, device="cuda") -> torch.Tensor:
    """A zeroed workspace for the spd_pages_* calls over pools of num_pages pages, and for every other call of the shape but the *_drafted ones."""
    return torch.zeros(spd_pages_workspace_size(shape, num_pages), dtype=torch.uint8, device=device)


def spd_pages_take(shape, refs, page_indptr, page_indices, from_tokens, to_tokens, ws, stream=None) -> None:
    """Fresh pages for the entries of tokens [from_tokens[u], to_tokens[u]) that hold -1 (int32 [B] each)."""
    dev, n, B = _here(refs), refs.numel(), shape.batch
    _check(lib().spd_pages_take(shape, n, _ints(refs, n, dev), _ints(page_indptr, B + 1, dev), _ints(page_indices, page_indices.numel(), dev),
                                _ints(from_tokens, B, dev), _ints(to_tokens, B, dev), *_workspace(ws, dev), _stream_ptr(stream)), "spd_pages_take")


def spd_pages_release(shape, refs, page_indptr, page_indices, from_tokens, ws, to_tokens=None, stream=None) -> None:
    """Take the entries that hold nothing but tokens [from_tokens[u], to_tokens[u]) out of the tables; to_tokens None: to the tables' end."""
    dev, n, B = _here(refs), refs.numel(), shape.batch
    _check(lib().spd_pages_release(shape, n, _ints(refs, n, dev), _ints(page_indptr, B + 1, dev), _ints(page_indices, page_indices.numel(), dev),
                                   _ints(from_tokens, B, dev), _ints(to_tokens, B, dev), *_workspace(ws, dev), _stream_ptr(stream)), "spd_pages_release")


def spd_pages_fork(shape, refs, page_indptr, page_indices, seq_lens, source, copies, ws, stream=None) -> None:
    """User u becomes a copy of user source[u] (int32 [B], -1: it stays); copies int32 [B, 2] receives the pages to copy (spd_pages_copy)."""
    dev, n, B = _here(refs), refs.numel(), shape.batch
    _check(lib().spd_pages_fork(shape, n, _ints(refs, n, dev), _ints(page_indptr, B + 1, dev), _ints(page_indices, page_indices.numel(), dev),
                                _ints(seq_lens, B, dev), _ints(source, B, dev), _ints(copies, 2 * B, dev), *_workspace(ws, dev),
                                _stream_ptr(stream)), "spd_pages_fork")


def spd_pages_copy(shape, pools, copies, ws, stream=None) -> None:
    """Copy page copies[i, 0] to page copies[i, 1] (int32 [n, 2]) in all pools (make_pools, or a list of tensors)."""
    dev = _here(copies)
    pools, n = _pools(shape, pools, dev), copies.shape[0]
    _check(lib().spd_pages_copy(shape, pools.count, pools.array, pools.pages, n, _ints(copies, 2 * n, dev), *_workspace(ws, dev),
                                _stream_ptr(stream)), "spd_pages_copy")
