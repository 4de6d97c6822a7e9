"""MI355X-native segment re-prefill: Python binding of the C ABI in include/sa.h.

The binding only marshals arguments: torch tensors supply device pointers and
the current HIP stream, host length arrays are converted to int32, and every
computation happens in the HIP kernels of ``libsa.so``.  If the library is not
built, importing works but every call raises -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

__all__ = [
    "Layout", "Context", "SaError", "library_path", "load_library",
    "sa_kv_append", "sa_kv_assemble", "sa_kv_assemble_append", "sa_kv_splice_alias",
    "sa_segment_prefill_attn", "sa_segment_prefill_attn_append", "sa_set_exact_scale", "sa_set_fused_append",
    "sa_set_kernel_events", "sa_set_block_clock", "sa_set_xcd_weights", "sa_sync_check", "sa_reserve",
    "sa_segment_prefill_attn_noalloc", "sa_attn_plan_stats", "Rope", "sa_kv_append_rope", "sa_kv_fork",
    "sa_kv_retain", "sa_kv_release", "sa_kv_compact", "sa_shared_prefix_attn", "sa_shared_plan_stats",
    "sa_kv_append_rope_axes", "kvq_pool_shape", "sa_kvq_append", "sa_kvq_pack", "sa_kvq_unpack", "sa_kvq_attn",
    "EXPORTED_SYMBOLS",
]

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libsa.so")
_lib = None

EXPORTED_SYMBOLS = ("sa_create", "sa_destroy", "sa_status_string", "sa_last_error",
                    "sa_sync_check", "sa_kv_append", "sa_kv_assemble", "sa_kv_assemble_append",
                    "sa_kv_splice_alias", "sa_segment_prefill_attn", "sa_segment_prefill_attn_append",
                    "sa_set_exact_scale", "sa_set_fused_append", "sa_set_kernel_events",
                    "sa_set_block_clock", "sa_set_xcd_weights", "sa_reserve",
                    "sa_segment_prefill_attn_noalloc", "sa_attn_plan_stats", "sa_kv_append_rope",
                    "sa_kv_fork", "sa_kv_retain", "sa_kv_release", "sa_kv_compact", "sa_shared_prefix_attn",
                    "sa_shared_plan_stats", "sa_kv_append_rope_axes", "sa_kvq_append", "sa_kvq_pack",
                    "sa_kvq_unpack", "sa_kvq_attn")

STATUS = {0: "SA_OK", 1: "SA_ERR_NULL", 2: "SA_ERR_SHAPE", 3: "SA_ERR_UNSUPPORTED",
          4: "SA_ERR_ALIGN", 5: "SA_ERR_RANGE", 6: "SA_ERR_NO_PAGES", 7: "SA_ERR_HIP",
          8: "SA_ERR_DEVICE", 9: "SA_ERR_OVERLAP"}


class SaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status
        self.name = STATUS.get(status, str(status))


class Layout(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_layers", ctypes.c_int32), ("num_slots", ctypes.c_int64)]


class _Pages(ctypes.Structure):
    _fields_ = [("indptr", ctypes.c_void_p), ("indices", ctypes.c_void_p)]


class _Rope(ctypes.Structure):
    _fields_ = [("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("h_inv_freq", ctypes.c_void_p),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float),
                ("weight_offset", ctypes.c_float)]


class _Axes(ctypes.Structure):
    _fields_ = [("num_axes", ctypes.c_int32), ("h_axis", ctypes.c_void_p), ("d_pos", ctypes.c_void_p),
                ("pos_stride", ctypes.c_int64)]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load libsa.so; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is not built; run paper_2607_00151_amd.build.build()")
    lib = ctypes.CDLL(_LIB_PATH)
    P, I32, I64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
    LP = ctypes.POINTER(Layout)
    lib.sa_create.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_void_p)]
    lib.sa_destroy.argtypes = [P]
    lib.sa_destroy.restype = None
    lib.sa_status_string.argtypes = [ctypes.c_int]
    lib.sa_status_string.restype = ctypes.c_char_p
    lib.sa_last_error.argtypes = []
    lib.sa_last_error.restype = ctypes.c_char_p
    lib.sa_sync_check.argtypes = [P, P]
    lib.sa_kv_append.argtypes = [P, LP, I32, P, P, P, P, I32, P, P, _Pages, P]
    lib.sa_kv_assemble.argtypes = [P, LP, P, P, P, P, I32, P, P, P, P, _Pages, P, I32, P, P, I32,
                                   P, P]
    lib.sa_kv_assemble_append.argtypes = [P, LP, P, P, P, P, I32, P, P, P, P, _Pages, P, I32, P, P, I32,
                                          P, I32, P, P, P, P]
    lib.sa_kv_splice_alias.argtypes = [P, LP, I32, P, P, P, P, _Pages, P, I32, P, P, I32, P, P]
    lib.sa_segment_prefill_attn.argtypes = [P, LP, I32, P, P, P, I32, P, P, _Pages, ctypes.c_float,
                                            P, P, P]
    lib.sa_segment_prefill_attn_append.argtypes = [P, LP, I32, P, P, P, P, P, I32, P, P, _Pages,
                                                   ctypes.c_float, P, P, P]
    lib.sa_set_exact_scale.argtypes = [P, I32]
    lib.sa_set_fused_append.argtypes = [P, I32]
    lib.sa_set_kernel_events.argtypes = [P, I32, P, P]
    lib.sa_set_block_clock.argtypes = [P, P, I64, ctypes.POINTER(ctypes.c_int64)]
    lib.sa_set_xcd_weights.argtypes = [P, P]
    lib.sa_reserve.argtypes = [P, I64, I64]
    lib.sa_segment_prefill_attn_noalloc.argtypes = lib.sa_segment_prefill_attn.argtypes
    lib.sa_attn_plan_stats.argtypes = [LP, I32, P, P, I32, P]
    lib.sa_kv_append_rope.argtypes = [P, LP, I32, ctypes.POINTER(_Rope), P, I64, P, I64, P, I64, P, P, P, I32, P, P,
                                      P, _Pages, P]
    lib.sa_kv_fork.argtypes = [P, LP, P, P, I32, P, I32, P, P, _Pages, P, I32, P, P, I32, P, P, P]
    lib.sa_kv_retain.argtypes = [P, LP, I32, _Pages, I64, P, P]
    lib.sa_kv_release.argtypes = [P, LP, I32, _Pages, I64, P, P, P, P]
    lib.sa_kv_compact.argtypes = [P, LP, P, P, I32, P, P, P, P, I64, P, P, P]
    lib.sa_shared_prefix_attn.argtypes = [P, LP, I32, P, P, P, I32, P, P, _Pages, I32, P, P, ctypes.c_float, P, P, P]
    lib.sa_shared_plan_stats.argtypes = [LP, I32, P, P, I32, P, P, I32, P, P]
    RP, AP = ctypes.POINTER(_Rope), ctypes.POINTER(_Axes)
    lib.sa_kv_append_rope_axes.argtypes = [P, LP, I32, RP, AP, P, I64, P, I64, P, I64, P, P, P, I32, P, P, _Pages, P]
    lib.sa_kvq_append.argtypes = [P, LP, I32, RP, AP, P, I64, P, I64, P, I64, P, P, P, I32, P, P, P, _Pages, P]
    lib.sa_kvq_pack.argtypes = [P, LP, P, P, P, I64, P, P, P, I32, P]
    lib.sa_kvq_unpack.argtypes = [P, LP, I64, P, P, P, P, P, P, I32, P]
    lib.sa_kvq_attn.argtypes = [P, LP, I32, P, P, P, I32, P, P, _Pages, I32, ctypes.c_float, P, P, P]
    for name in ("sa_create", "sa_sync_check", "sa_kv_append", "sa_kv_assemble", "sa_kv_assemble_append",
                 "sa_kv_splice_alias", "sa_segment_prefill_attn", "sa_segment_prefill_attn_append",
                 "sa_set_exact_scale", "sa_set_fused_append", "sa_set_kernel_events", "sa_set_block_clock",
                 "sa_set_xcd_weights",
                 "sa_reserve", "sa_segment_prefill_attn_noalloc", "sa_attn_plan_stats", "sa_kv_append_rope",
                 "sa_kv_fork", "sa_kv_retain", "sa_kv_release", "sa_kv_compact", "sa_shared_prefix_attn",
                 "sa_shared_plan_stats", "sa_kv_append_rope_axes", "sa_kvq_append", "sa_kvq_pack", "sa_kvq_unpack",
                 "sa_kvq_attn"):
        getattr(lib, name).restype = ctypes.c_int
    _lib = lib
    return lib


_byte_of = ctypes.c_char.from_buffer
_addressof = ctypes.addressof


def _check(status: int):
    if status != 0:
        msg = load_library().sa_last_error().decode(errors="replace")
        raise SaError(status, msg)


def _ptr(t):
    """Address of a host numpy array, or None."""
    if t is None:
        return None
    try:
        return _addressof(_byte_of(t))         # a quarter of the time of ndarray.ctypes, 1 us of every array of a call
    except (TypeError, ValueError):            # read-only or empty
        return t.ctypes.data


_torch = None
_KINDS = None
_raw_stream = None


def _load_torch():
    global _torch, _KINDS, _raw_stream
    import torch
    two = {d for d in (getattr(torch, n, None) for n in ("bfloat16", "float16", "int16", "uint16")) if d is not None}
    _KINDS = {"i32": {torch.int32}, "b16": two, "f32": {torch.float32}, "u8": {torch.uint8}, "bf16": two - {torch.float16}}
    # the current stream's handle without a Stream object around it, where torch has it
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _torch = torch
    return torch


def _dev(t, what: str, kind: str, min_numel: int = 0, nullable: bool = False):
    """Device address of a caller tensor after checking what the C ABI will assume
    of it: a contiguous CUDA tensor whose element type matches `kind` ("i32": int32
    table entries, "b16": 2-byte bf16 bit patterns, "bf16": the same, but not
    float16, "f32": float32) and that holds at
    least min_numel elements.  Raises ValueError otherwise; None passes only when
    nullable."""
    if t is None:
        if nullable:
            return None
        raise ValueError(f"{what}: a device tensor is required")
    torch = _torch or _load_torch()
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{what}: expected a torch tensor, got {type(t).__name__}")
    if not t.is_cuda:
        raise ValueError(f"{what}: tensor is not on a GPU")
    if not t.is_contiguous():
        raise ValueError(f"{what}: tensor is not contiguous")
    # the types in everyday use by a table; any other 2-byte type that is not bool by its size
    if t.dtype not in _KINDS[kind] and not (kind == "b16" and t.element_size() == 2 and t.dtype != torch.bool):
        want = {"i32": "torch.int32", "b16": "a 2-byte dtype (bf16 bits)", "f32": "torch.float32",
                "bf16": "torch.bfloat16 (or its bits in a 2-byte integer)", "u8": "torch.uint8"}[kind]
        raise ValueError(f"{what}: dtype {t.dtype}, expected {want}")
    if t.numel() < min_numel:
        raise ValueError(f"{what}: {t.numel()} elements, at least {min_numel} needed")
    return t.data_ptr() or None


def _pool_numel(layout) -> int:
    return (int(layout.num_layers) * int(layout.num_slots) * int(layout.num_kv_heads)
            * int(layout.page_size) * int(layout.head_dim))


_I32 = np.dtype(np.int32)


def _host_i32(x):
    # an aligned int32 array is read where it is (within the call); anything else is converted and range-checked
    if type(x) is np.ndarray and x.dtype == _I32 and x.flags.c_contiguous and x.flags.aligned and x.ndim > 0:
        return x
    a = np.ascontiguousarray(np.asarray(x, dtype=np.int64))
    if a.size and (a.min() < -2**31 or a.max() >= 2**31):
        raise OverflowError("value does not fit int32")
    return np.ascontiguousarray(a, dtype=np.int32)


def _total(a) -> int:
    """Sum of a host int32 array, in Python's integers (numpy's reduction costs more on a short one)."""
    return sum(a.tolist()) if a.size <= 64 and a.ndim == 1 else int(a.sum(dtype=np.int64))


def _stream(stream):
    if stream is None:
        torch = _torch or _load_torch()
        if _raw_stream is not None:
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if hasattr(stream, "cuda_stream"):
        return stream.cuda_stream
    return int(stream)


def _pages(indptr, indices, batch: int, what: str = "page table"):
    return _Pages(_dev(indptr, f"{what} indptr", "i32", batch + 1),
                  _dev(indices, f"{what} indices", "i32", 0))


class Context:
    """Owns an sa_ctx (plan buffers, staging, split scratch) on one device."""

    def __init__(self, device: int = 0):
        lib = load_library()
        h = ctypes.c_void_p()
        _check(lib.sa_create(int(device), ctypes.byref(h)))
        self._h = h
        self.device = device

    @property
    def handle(self):
        return self._h

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            load_library().sa_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def _ctx_handle(ctx):
    if ctx is None:
        return None
    return ctx.handle if isinstance(ctx, Context) else ctx


def sa_reserve(ctx, plan_bytes: int, split_bytes: int = 0):
    """Size ctx's plan buffers (each call kind's, the pinned staging and the slot scans' buffer) to
    plan_bytes and its split-KV partials to split_bytes, so later calls that fit allocate nothing."""
    _check(load_library().sa_reserve(_ctx_handle(ctx), int(plan_bytes), int(split_bytes)))


def sa_attn_plan_stats(layout: Layout, q_len, kv_len, num_cu: int = 256) -> dict:
    """Shape of the attention launch these lengths make (host only, no GPU): workgroups,
    split parts, 64-key tiles and the makespan in tiles over 2 x num_cu slots."""
    q_len, kv_len = _host_i32(q_len), _host_i32(kv_len)
    if q_len.shape != kv_len.shape:
        raise ValueError("q_len and kv_len differ in length")
    out = np.zeros(4, dtype=np.int64)
    _check(load_library().sa_attn_plan_stats(ctypes.byref(layout), int(len(q_len)), _ptr(q_len), _ptr(kv_len),
                                             int(num_cu), out.ctypes.data))
    return {"items": int(out[0]), "parts": int(out[1]), "tiles": int(out[2]), "makespan_tiles": int(out[3])}


def sa_sync_check(ctx, stream=None):
    _check(load_library().sa_sync_check(_ctx_handle(ctx), _stream(stream)))


def sa_kv_append(ctx, layout: Layout, layer: int, k_pool, v_pool, k_new, v_new, start, new_len,
                 pages_indptr, pages_indices, stream=None):
    start, new_len = _host_i32(start), _host_i32(new_len)
    if start.shape != new_len.shape:
        raise ValueError("start and new_len differ in length")
    B = len(new_len)
    rows = _total(new_len) * int(layout.num_kv_heads) * int(layout.head_dim)
    _check(load_library().sa_kv_append(
        _ctx_handle(ctx), ctypes.byref(layout), int(layer),
        _dev(k_pool, "k_pool", "b16", _pool_numel(layout)), _dev(v_pool, "v_pool", "b16", _pool_numel(layout)),
        _dev(k_new, "k_new", "b16", rows, nullable=rows == 0), _dev(v_new, "v_new", "b16", rows, nullable=rows == 0),
        int(B), _ptr(start), _ptr(new_len), _pages(pages_indptr, pages_indices, B), _stream(stream)))


def _splice_host(layout, src_len, keep_indptr, keep_spans, reserve):
    src_len, reserve = _host_i32(src_len), _host_i32(reserve)
    keep_indptr = _host_i32(keep_indptr)
    keep_spans = _host_i32(np.asarray(keep_spans).reshape(-1))
    B = len(src_len)
    if len(reserve) != B or len(keep_indptr) != B + 1:
        raise ValueError("per-sequence arrays disagree on the batch size")
    return src_len, keep_indptr, keep_spans, reserve, B


def _splice_dev(layout, B, k_src, v_src, k_dst, v_dst, src_indptr, src_indices, fresh, dst_indptr,
                dst_indices, fresh_nullable=False):
    n = _pool_numel(layout)
    return (_dev(k_src, "k_src", "b16", n), _dev(v_src, "v_src", "b16", n),
            _dev(k_dst, "k_dst", "b16", n), _dev(v_dst, "v_dst", "b16", n),
            _Pages(_dev(src_indptr, "src indptr", "i32", B + 1),
                   _dev(src_indices, "src indices", "i32", 0, nullable=True)),
            _dev(fresh, "fresh", "i32", 0, nullable=fresh_nullable),
            0 if fresh is None else int(fresh.numel()),
            _dev(dst_indptr, "dst indptr", "i32", B + 1),
            _dev(dst_indices, "dst indices", "i32", 0, nullable=True),
            0 if dst_indices is None else int(dst_indices.numel()))


def sa_kv_assemble(ctx, layout: Layout, k_src, v_src, k_dst, v_dst, src_len, keep_indptr,
                   keep_spans, reserve, src_indptr, src_indices, fresh, dst_indptr, dst_indices,
                   stream=None):
    """Returns the kept token count of every sequence (numpy int32)."""
    src_len, keep_indptr, keep_spans, reserve, B = _splice_host(layout, src_len, keep_indptr, keep_spans,
                                                                reserve)
    ks, vs, kd, vd, src, fr, nfr, dip, dix, cap = _splice_dev(layout, B, k_src, v_src, k_dst, v_dst,
                                                              src_indptr, src_indices, fresh, dst_indptr,
                                                              dst_indices)
    dst_len = np.zeros(B, dtype=np.int32)
    _check(load_library().sa_kv_assemble(
        _ctx_handle(ctx), ctypes.byref(layout), ks, vs, kd, vd, B, _ptr(src_len), _ptr(keep_indptr),
        _ptr(keep_spans) if keep_spans.size else None, _ptr(reserve), src, fr, nfr, dip, dix, cap,
        _ptr(dst_len), _stream(stream)))
    return dst_len


def sa_kv_assemble_append(ctx, layout: Layout, k_src, v_src, k_dst, v_dst, src_len, keep_indptr,
                          keep_spans, reserve, src_indptr, src_indices, fresh, dst_indptr, dst_indices,
                          layer, k_new, v_new, new_len, stream=None):
    """Splice and the segment's append in one launch.  Returns the kept token
    count of every sequence (numpy int32); the new rows follow it."""
    src_len, keep_indptr, keep_spans, reserve, B = _splice_host(layout, src_len, keep_indptr, keep_spans,
                                                                reserve)
    new_len = _host_i32(new_len)
    if len(new_len) != B:
        raise ValueError("per-sequence arrays disagree on the batch size")
    ks, vs, kd, vd, src, fr, nfr, dip, dix, cap = _splice_dev(layout, B, k_src, v_src, k_dst, v_dst,
                                                              src_indptr, src_indices, fresh, dst_indptr,
                                                              dst_indices)
    rows = _total(new_len) * int(layout.num_kv_heads) * int(layout.head_dim)
    dst_len = np.zeros(B, dtype=np.int32)
    _check(load_library().sa_kv_assemble_append(
        _ctx_handle(ctx), ctypes.byref(layout), ks, vs, kd, vd, B, _ptr(src_len), _ptr(keep_indptr),
        _ptr(keep_spans) if keep_spans.size else None, _ptr(reserve), src, fr, nfr, dip, dix, cap,
        _ptr(dst_len), int(layer), _dev(k_new, "k_new", "b16", rows, nullable=rows == 0),
        _dev(v_new, "v_new", "b16", rows, nullable=rows == 0), _ptr(new_len), _stream(stream)))
    return dst_len


def sa_kv_splice_alias(ctx, layout: Layout, src_len, keep_indptr, keep_spans, reserve, src_indptr,
                       src_indices, fresh, dst_indptr, dst_indices, stream=None):
    """Zero-copy splice: the destination table shares the surviving source slots.
    Returns the kept token count of every sequence (numpy int32)."""
    src_len, keep_indptr, keep_spans, reserve, B = _splice_host(layout, src_len, keep_indptr, keep_spans,
                                                                reserve)
    dst_len = np.zeros(B, dtype=np.int32)
    _check(load_library().sa_kv_splice_alias(
        _ctx_handle(ctx), ctypes.byref(layout), B, _ptr(src_len), _ptr(keep_indptr),
        _ptr(keep_spans) if keep_spans.size else None, _ptr(reserve),
        _Pages(_dev(src_indptr, "src indptr", "i32", B + 1),
               _dev(src_indices, "src indices", "i32", 0, nullable=True)),
        _dev(fresh, "fresh", "i32", 0, nullable=True), 0 if fresh is None else int(fresh.numel()),
        _dev(dst_indptr, "dst indptr", "i32", B + 1), _dev(dst_indices, "dst indices", "i32", 0, nullable=True),
        0 if dst_indices is None else int(dst_indices.numel()), _ptr(dst_len), _stream(stream)))
    return dst_len


def _attn_dev(layout, q_len, q, o, lse):
    T = _total(q_len)
    n = T * int(layout.num_q_heads) * int(layout.head_dim)
    return (_dev(q, "q", "b16", n, nullable=T == 0), _dev(o, "o", "b16", n, nullable=T == 0),
            _dev(lse, "lse", "f32", T * int(layout.num_q_heads), nullable=True), T)


def sa_segment_prefill_attn(ctx, layout: Layout, layer: int, q, k_pool, v_pool, q_len, kv_len,
                            pages_indptr, pages_indices, softmax_scale: float, o, lse=None,
                            stream=None):
    q_len, kv_len = _host_i32(q_len), _host_i32(kv_len)
    if q_len.shape != kv_len.shape:
        raise ValueError("q_len and kv_len differ in length")
    qp, op, lp, _ = _attn_dev(layout, q_len, q, o, lse)
    n = _pool_numel(layout)
    _check(load_library().sa_segment_prefill_attn(
        _ctx_handle(ctx), ctypes.byref(layout), int(layer), qp, _dev(k_pool, "k_pool", "b16", n),
        _dev(v_pool, "v_pool", "b16", n), int(len(q_len)), _ptr(q_len), _ptr(kv_len),
        _pages(pages_indptr, pages_indices, len(q_len)), float(softmax_scale), op, lp, _stream(stream)))


def sa_segment_prefill_attn_noalloc(ctx, layout: Layout, layer: int, q, k_pool, v_pool, q_len, kv_len,
                                    pages_indptr, pages_indices, softmax_scale: float, o, lse=None, stream=None):
    """sa_segment_prefill_attn without any device allocation: plan and split partials in the
    library's fixed per-GPU scratch array (calls on one GPU must not overlap in time)."""
    q_len, kv_len = _host_i32(q_len), _host_i32(kv_len)
    if q_len.shape != kv_len.shape:
        raise ValueError("q_len and kv_len differ in length")
    qp, op, lp, _ = _attn_dev(layout, q_len, q, o, lse)
    n = _pool_numel(layout)
    _check(load_library().sa_segment_prefill_attn_noalloc(
        _ctx_handle(ctx), ctypes.byref(layout), int(layer), qp, _dev(k_pool, "k_pool", "b16", n),
        _dev(v_pool, "v_pool", "b16", n), int(len(q_len)), _ptr(q_len), _ptr(kv_len),
        _pages(pages_indptr, pages_indices, len(q_len)), float(softmax_scale), op, lp, _stream(stream)))


def sa_set_exact_scale(ctx, enable: bool = True):
    """Later attention calls on ctx apply the softmax scale to each score in fp32
    (enable, the default) or fold it into the bf16 query rows."""
    _check(load_library().sa_set_exact_scale(_ctx_handle(ctx), int(bool(enable))))


def sa_set_fused_append(ctx, enable: bool = True):
    """Later sa_segment_prefill_attn_append calls on ctx write the segment's rows
    inside the attention launch (enable) or with an append launch before it (the
    default)."""
    _check(load_library().sa_set_fused_append(_ctx_handle(ctx), int(bool(enable))))


def sa_set_block_clock(ctx, buf=None) -> int:
    """Later launches of the default attention kernel on ctx write, per workgroup,
    four int64 words into buf (a device int64 tensor of 4 x max workgroups):
    start and end clock, sequence, q_len.  Returns the clock's rate in kHz.
    None clears."""
    khz = ctypes.c_int64(0)
    if buf is not None and (not hasattr(buf, "element_size") or buf.element_size() != 8 or not buf.is_cuda
                            or not buf.is_contiguous()):
        raise ValueError("sa_set_block_clock needs a contiguous device tensor of 8-byte elements")
    n = 0 if buf is None else buf.numel() // 4
    _check(load_library().sa_set_block_clock(_ctx_handle(ctx), None if buf is None else buf.data_ptr(), n,
                                             ctypes.byref(khz)))
    return int(khz.value)


def sa_set_xcd_weights(ctx, speeds=None):
    """Relative speeds of the 8 XCDs for the attention planner (None: equal)."""
    if speeds is None:
        _check(load_library().sa_set_xcd_weights(_ctx_handle(ctx), None))
        return
    w = np.ascontiguousarray(speeds, dtype=np.float32)
    if w.shape != (8,):
        raise ValueError("sa_set_xcd_weights needs 8 speeds")
    _check(load_library().sa_set_xcd_weights(_ctx_handle(ctx), w.ctypes.data))


TIMED_ATTN, TIMED_PAGES = 0, 1


def sa_set_kernel_events(ctx, which: int, start_event=None, stop_event=None):
    """Later kernels of kind `which` (TIMED_ATTN, TIMED_PAGES) on ctx are launched
    bound to these two hipEvent_t handles (ints), which then time the kernel
    itself; None, None clears."""
    _check(load_library().sa_set_kernel_events(_ctx_handle(ctx), int(which), start_event or None,
                                               stop_event or None))


def sa_segment_prefill_attn_append(ctx, layout: Layout, layer: int, q, k_pool, v_pool, k_new, v_new, q_len,
                                   kv_len, pages_indptr, pages_indices, softmax_scale: float, o, lse=None,
                                   stream=None):
    """Writes each sequence's q_len new K/V rows at positions kv_len - q_len .. kv_len - 1,
    then runs sa_segment_prefill_attn over the result."""
    q_len, kv_len = _host_i32(q_len), _host_i32(kv_len)
    if q_len.shape != kv_len.shape:
        raise ValueError("q_len and kv_len differ in length")
    qp, op, lp, T = _attn_dev(layout, q_len, q, o, lse)
    rows = T * int(layout.num_kv_heads) * int(layout.head_dim)
    n = _pool_numel(layout)
    _check(load_library().sa_segment_prefill_attn_append(
        _ctx_handle(ctx), ctypes.byref(layout), int(layer), qp, _dev(k_pool, "k_pool", "b16", n),
        _dev(v_pool, "v_pool", "b16", n), _dev(k_new, "k_new", "b16", rows, nullable=T == 0),
        _dev(v_new, "v_new", "b16", rows, nullable=T == 0), int(len(q_len)), _ptr(q_len), _ptr(kv_len),
        _pages(pages_indptr, pages_indices, len(q_len)), float(softmax_scale), op, lp, _stream(stream)))


# ---------------------------------------------------------------- branches of one context

def _device_of(ctx):
    """ctx's device, or None where it is only a handle."""
    return ctx.device if isinstance(ctx, Context) else None


def _on(t, what: str, kind: str, min_numel: int, device, nullable: bool = False):
    """_dev for the branch calls, which run on ctx's device: a tensor elsewhere is refused rather than read there.
    One pass of the cheap tests for the usual case; _dev names what is wrong with any other."""
    try:
        at = t.get_device()
        if at == device and t.dtype in _KINDS[kind] and t.is_contiguous() and t.numel() >= min_numel:
            return t.data_ptr() or None
    except (AttributeError, TypeError):        # no tensor, or the first call
        at = -1
    if at >= 0 and device is not None and at != device:
        raise ValueError(f"{what}: the tensor is on device {at}, the context on device {device}")
    return _dev(t, what, kind, min_numel, nullable)


def _stream_of(ctx, stream):
    """`stream`, or torch's current stream of ctx's device (not of the current device)."""
    if stream is None and isinstance(ctx, Context):
        torch = _torch or _load_torch()
        if _raw_stream is not None:
            return _raw_stream(ctx.device)
        return torch.cuda.current_stream(ctx.device).cuda_stream
    return _stream(stream)


def _head_rows(t, what: str, tokens: int, heads: int, d: int, device):
    """(address, token stride in elements) of a [tokens][heads][d] tensor whose heads are contiguous within a token."""
    if tokens == 0:
        return (None if t is None else t.data_ptr() or None), heads * d
    torch = _torch or _load_torch()
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{what}: a device tensor is required")
    at = t.get_device()
    if at < 0:
        raise ValueError(f"{what}: tensor is not on a GPU")
    if device is not None and at != device:
        raise ValueError(f"{what}: the tensor is on device {at}, the context on device {device}")
    if t.dtype not in _KINDS["bf16"]:
        raise ValueError(f"{what}: dtype {t.dtype}, expected torch.bfloat16 (or its bits in a 2-byte integer)")
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[0] < tokens or shape[1] != heads or shape[2] != d:
        raise ValueError(f"{what}: shape {tuple(shape)}, expected ({tokens}, {heads}, {d})")
    if stride[2] != 1 or (heads > 1 and stride[1] != d):
        raise ValueError(f"{what}: the heads of a token must be contiguous")
    return t.data_ptr(), stride[0] if shape[0] > 1 else heads * d


class Rope:
    """Norms and rotation of sa_kv_append_rope (sa_rope): inv_freq, radians per position of each pair of dims
    (float64, its length sets rot_dim); q_weight, k_weight, bf16 norm weights of one head (None: no norm)."""

    def __init__(self, inv_freq=(), q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False,
                 weight_offset: float = 0.0):
        self.inv_freq = inv_freq
        self.q_weight, self.k_weight = q_weight, k_weight
        self.eps, self.interleaved, self.weight_offset = float(eps), bool(interleaved), float(weight_offset)

    @property
    def inv_freq(self):
        return self._inv_freq

    @inv_freq.setter
    def inv_freq(self, value):                 # read as doubles by every call, whatever it is set from
        self._inv_freq = np.ascontiguousarray(value, dtype=np.float64).reshape(-1)

    def _struct(self, d: int, device):
        n = len(self._inv_freq)
        return _Rope(2 * n, self.interleaved, _ptr(self._inv_freq) if n else None,
                     None if self.q_weight is None else _on(self.q_weight, "q_weight", "bf16", d, device),
                     None if self.k_weight is None else _on(self.k_weight, "k_weight", "bf16", d, device), self.eps,
                     self.weight_offset)


def sa_kv_append_rope(ctx, layout: Layout, layer: int, rope: Rope, q, k_new, v_new, q_out, k_pool, v_pool, start,
                      new_len, pages_indptr, pages_indices, pos=None, stream=None):
    """Norms and rotates the query and key heads of new tokens; query rows go to q_out, key and value rows into
    their pages.  q, k_new, v_new: [tokens][heads][128], possibly slices of one projection's output.  pos: rotation
    position of each sequence's first new token (None: start)."""
    start, new_len = _host_i32(start), _host_i32(new_len)
    pos = None if pos is None else _host_i32(pos)
    if start.shape != new_len.shape or (pos is not None and pos.shape != start.shape):
        raise ValueError("start, new_len and pos differ in length")
    B, T, D, at = len(new_len), max(0, _total(new_len)), layout.head_dim, _device_of(ctx)
    Hq, Hkv = layout.num_q_heads, layout.num_kv_heads
    qp, qs = _head_rows(q, "q", T, Hq, D, at)
    kp, ks = _head_rows(k_new, "k_new", T, Hkv, D, at)
    vp, vs = _head_rows(v_new, "v_new", T, Hkv, D, at)
    n = _pool_numel(layout)
    _check(load_library().sa_kv_append_rope(
        _ctx_handle(ctx), ctypes.byref(layout), int(layer), ctypes.byref(rope._struct(D, at)), qp, qs, kp, ks, vp, vs,
        _on(q_out, "q_out", "bf16", T * Hq * D, at, nullable=T == 0), _on(k_pool, "k_pool", "bf16", n, at),
        _on(v_pool, "v_pool", "bf16", n, at), B, _ptr(start), _ptr(new_len), _ptr(pos),
        _table_on(pages_indptr, pages_indices, B, at, "page table"), _stream_of(ctx, stream)))


def _table_on(indptr, indices, batch: int, device, what: str, nullable: bool = False):
    return _Pages(_on(indptr, f"{what} indptr", "i32", batch + 1, device),
                  _on(indices, f"{what} indices", "i32", 0, device, nullable))


def sa_kv_fork(ctx, layout: Layout, k_pool, v_pool, src_len, parent, reserve, src_indptr, src_indices, fresh,
               dst_indptr, dst_indices, ref=None, stream=None) -> int:
    """Opens children of cached contexts: shared full pages, a copy of the partial one, fresh pages for reserve.
    parent: the sequence each child continues.  Returns the number of fresh slots taken."""
    src_len, parent, reserve = _host_i32(src_len), _host_i32(parent), _host_i32(reserve)
    if parent.shape != reserve.shape:
        raise ValueError("parent and reserve differ in length")
    B, C, n, at = len(src_len), len(parent), _pool_numel(layout), _device_of(ctx)
    used = ctypes.c_int32(0)
    _check(load_library().sa_kv_fork(
        _ctx_handle(ctx), ctypes.byref(layout), _on(k_pool, "k_pool", "bf16", n, at), _on(v_pool, "v_pool", "bf16", n, at),
        B, _ptr(src_len), C, _ptr(parent), _ptr(reserve), _table_on(src_indptr, src_indices, B, at, "src", True),
        _on(fresh, "fresh", "i32", 0, at, nullable=True), 0 if fresh is None else fresh.numel(),
        _on(dst_indptr, "dst indptr", "i32", C + 1, at), _on(dst_indices, "dst indices", "i32", 0, at, nullable=True),
        0 if dst_indices is None else dst_indices.numel(),
        _on(ref, "ref", "i32", layout.num_slots, at, nullable=True), ctypes.addressof(used), _stream_of(ctx, stream)))
    return used.value


def _count_args(ctx, layout, pages_indptr, pages_indices, ref):
    at = _device_of(ctx)
    table = _table_on(pages_indptr, pages_indices, 1, at, "page table")
    return (_ctx_handle(ctx), ctypes.byref(layout), pages_indptr.numel() - 1, table, pages_indices.numel(),
            _on(ref, "ref", "i32", layout.num_slots, at))


def sa_kv_retain(ctx, layout: Layout, pages_indptr, pages_indices, ref, stream=None):
    """Raises the count of every slot that the tables name."""
    _check(load_library().sa_kv_retain(*_count_args(ctx, layout, pages_indptr, pages_indices, ref),
                                       _stream_of(ctx, stream)))


def sa_kv_release(ctx, layout: Layout, pages_indptr, pages_indices, ref, free=None, num_free=None, stream=None):
    """Lowers the count of every slot that the tables name; free [num_slots] then lists the slots without a count,
    ascending, and num_free [1] says how many."""
    at = _device_of(ctx)
    _check(load_library().sa_kv_release(
        *_count_args(ctx, layout, pages_indptr, pages_indices, ref),
        _on(free, "free", "i32", layout.num_slots, at, nullable=True), _on(num_free, "num_free", "i32", 1, at, nullable=True),
        _stream_of(ctx, stream)))


def sa_kv_compact(ctx, layout: Layout, k_pool, v_pool, limit: int, ref, ref_out, indices, indices_out, slot_map, moved,
                  stream=None):
    """Moves the pages in use in slots >= limit into free slots below.  ref_out and indices_out may be ref and
    indices; slot_map [num_slots] receives where each slot's page is, moved [2] the pages moved and left."""
    n, slots, at = _pool_numel(layout), layout.num_slots, _device_of(ctx)
    entries = 0 if indices is None else indices.numel()
    _check(load_library().sa_kv_compact(
        _ctx_handle(ctx), ctypes.byref(layout), _on(k_pool, "k_pool", "bf16", n, at), _on(v_pool, "v_pool", "bf16", n, at),
        int(limit), _on(ref, "ref", "i32", slots, at), _on(ref_out, "ref_out", "i32", slots, at),
        _on(indices, "indices", "i32", 0, at, nullable=entries == 0),
        _on(indices_out, "indices_out", "i32", entries, at, nullable=entries == 0), entries,
        _on(slot_map, "slot_map", "i32", slots, at), _on(moved, "moved", "i32", 2, at), _stream_of(ctx, stream)))


def sa_shared_prefix_attn(ctx, layout: Layout, layer: int, q, k_pool, v_pool, q_len, kv_len, pages_indptr,
                          pages_indices, group_indptr, shared_len, softmax_scale: float, o, lse=None, stream=None):
    """sa_segment_prefill_attn for groups of sequences (group_indptr) that share their first shared_len tokens, whose
    keys and values are read once for the group."""
    q_len, kv_len = _host_i32(q_len), _host_i32(kv_len)
    groups, shared = _host_i32(group_indptr), _host_i32(shared_len)
    if q_len.shape != kv_len.shape:
        raise ValueError("q_len and kv_len differ in length")
    if len(groups) != len(shared) + 1:
        raise ValueError("group_indptr must have one entry more than shared_len")
    B, T, at, n = len(q_len), max(0, _total(q_len)), _device_of(ctx), _pool_numel(layout)
    rows = T * layout.num_q_heads
    _check(load_library().sa_shared_prefix_attn(
        _ctx_handle(ctx), ctypes.byref(layout), int(layer), _on(q, "q", "bf16", rows * layout.head_dim, at, T == 0),
        _on(k_pool, "k_pool", "bf16", n, at), _on(v_pool, "v_pool", "bf16", n, at), B, _ptr(q_len), _ptr(kv_len),
        _table_on(pages_indptr, pages_indices, B, at, "page table"), len(shared), _ptr(groups), _ptr(shared),
        float(softmax_scale), _on(o, "o", "bf16", rows * layout.head_dim, at, T == 0),
        None if lse is None else _on(lse, "lse", "f32", rows, at), _stream_of(ctx, stream)))


def sa_shared_plan_stats(layout: Layout, q_len, kv_len, group_indptr, shared_len, num_cu: int = 256) -> dict:
    """What sa_shared_prefix_attn would make of these lengths (host only, no GPU): which groups' prefixes are computed
    once (none: the batch goes to the segment attention), workgroups, rows of partial results, most parts of a row."""
    q_len, kv_len = _host_i32(q_len), _host_i32(kv_len)
    groups, shared = _host_i32(group_indptr), _host_i32(shared_len)
    if q_len.shape != kv_len.shape:
        raise ValueError("q_len and kv_len differ in length")
    if len(groups) != len(shared) + 1:
        raise ValueError("group_indptr must have one entry more than shared_len")
    out, once = np.zeros(4, dtype=np.int64), np.zeros(len(shared), dtype=np.int32)
    _check(load_library().sa_shared_plan_stats(
        ctypes.byref(layout), len(q_len), _ptr(q_len), _ptr(kv_len), len(shared), _ptr(groups), _ptr(shared),
        int(num_cu), out.ctypes.data, once.ctypes.data))
    return {"once": [bool(x) for x in once], "items": int(out[1]), "part_rows": int(out[2]), "most_parts": int(out[3])}


# ---------------------------------------------------------------- several axes, and a cache of 4 bits

_KVQ_ROW = 68            # bytes of a head row: 128 codes of 4 bits, 4 scale bytes


def kvq_pool_shape(layout: Layout):
    """Shape of one pool of 4 bits (torch.uint8) of this layout."""
    return (int(layout.num_layers), int(layout.num_slots), int(layout.num_kv_heads), int(layout.page_size) * _KVQ_ROW)


def _kvq_bytes(layout, slots) -> int:
    return int(layout.num_layers) * int(slots) * int(layout.num_kv_heads) * int(layout.page_size) * _KVQ_ROW


def _axes_of(rope, axis, pos, tokens: int, device):
    """(sa_axes, the host array it points to) of axis numbers [rot_dim / 2] and positions [num_axes][tokens]."""
    axis = _host_i32(axis)
    if axis.ndim != 1 or len(axis) != len(rope.inv_freq):
        raise ValueError(f"axis: {axis.shape}, expected one axis for each of the {len(rope.inv_freq)} frequencies")
    torch = _torch or _load_torch()
    if not isinstance(pos, torch.Tensor) or pos.dim() != 2:
        raise ValueError("pos: expected a device tensor [num_axes][tokens]")
    if pos.shape[1] < tokens:
        raise ValueError(f"pos: {pos.shape[1]} tokens, at least {tokens} needed")
    return _Axes(pos.shape[0], _ptr(axis) if len(axis) else None, _on(pos, "pos", "i32", 0, device), pos.shape[1]), axis


def sa_kv_append_rope_axes(ctx, layout: Layout, layer: int, rope: Rope, axis, q, k_new, v_new, q_out, k_pool, v_pool,
                           start, new_len, pages_indptr, pages_indices, pos, stream=None):
    """sa_kv_append_rope with a position per token and axis: pair j of token t turns by pos[axis[j], t] * inv_freq[j].
    axis: host integers, one for each frequency; pos: device int32 [num_axes][tokens]."""
    start, new_len = _host_i32(start), _host_i32(new_len)
    if start.shape != new_len.shape:
        raise ValueError("start and new_len differ in length")
    B, T, D, at = len(new_len), max(0, _total(new_len)), layout.head_dim, _device_of(ctx)
    Hq, Hkv = layout.num_q_heads, layout.num_kv_heads
    qp, qs = _head_rows(q, "q", T, Hq, D, at)
    kp, ks = _head_rows(k_new, "k_new", T, Hkv, D, at)
    vp, vs = _head_rows(v_new, "v_new", T, Hkv, D, at)
    axes, kept = _axes_of(rope, axis, pos, T, at)
    n = _pool_numel(layout)
    _check(load_library().sa_kv_append_rope_axes(
        _ctx_handle(ctx), ctypes.byref(layout), int(layer), ctypes.byref(rope._struct(D, at)), ctypes.byref(axes), qp,
        qs, kp, ks, vp, vs, _on(q_out, "q_out", "bf16", T * Hq * D, at, nullable=T == 0),
        _on(k_pool, "k_pool", "bf16", n, at), _on(v_pool, "v_pool", "bf16", n, at), B, _ptr(start), _ptr(new_len),
        _table_on(pages_indptr, pages_indices, B, at, "page table"), _stream_of(ctx, stream)))


def sa_kvq_append(ctx, layout: Layout, layer: int, k_new, v_new, kq_pool, vq_pool, start, new_len, pages_indptr,
                  pages_indices, rope: Rope = None, q=None, q_out=None, pos=None, axis=None, axis_pos=None, stream=None):
    """New key and value rows into pages of 4 bits.  With a rope the key heads, and the query heads of q (to q_out),
    are normed and rotated first: by pos (host, None: start), or by axis and axis_pos as in sa_kv_append_rope_axes."""
    start, new_len = _host_i32(start), _host_i32(new_len)
    pos = None if pos is None else _host_i32(pos)
    if start.shape != new_len.shape or (pos is not None and pos.shape != start.shape):
        raise ValueError("start, new_len and pos differ in length")
    if (axis is None) != (axis_pos is None):
        raise ValueError("axis and axis_pos go together")
    if rope is None and axis is not None:
        raise ValueError("axes without a rope")
    B, T, D, at = len(new_len), max(0, _total(new_len)), layout.head_dim, _device_of(ctx)
    Hq, Hkv = layout.num_q_heads, layout.num_kv_heads
    qp, qs = (None, 0) if q is None else _head_rows(q, "q", T, Hq, D, at)
    kp, ks = _head_rows(k_new, "k_new", T, Hkv, D, at)
    vp, vs = _head_rows(v_new, "v_new", T, Hkv, D, at)
    axes, kept = (None, None) if axis is None else _axes_of(rope, axis, axis_pos, T, at)
    n = _kvq_bytes(layout, layout.num_slots)
    _check(load_library().sa_kvq_append(
        _ctx_handle(ctx), ctypes.byref(layout), int(layer), None if rope is None else ctypes.byref(rope._struct(D, at)),
        None if axes is None else ctypes.byref(axes), qp, qs, kp, ks, vp, vs,
        None if q_out is None else _on(q_out, "q_out", "bf16", T * Hq * D, at), _on(kq_pool, "kq_pool", "u8", n, at),
        _on(vq_pool, "vq_pool", "u8", n, at), B, _ptr(start), _ptr(new_len), _ptr(pos),
        _table_on(pages_indptr, pages_indices, B, at, "page table"), _stream_of(ctx, stream)))


def _convert_args(ctx, layout, k_pool, v_pool, slots, kq_pool, vq_pool, slots4):
    at, n, page = _device_of(ctx), _pool_numel(layout), _kvq_bytes(layout, 1)
    pages = 0 if slots is None else slots.numel()
    if (0 if slots4 is None else slots4.numel()) != pages:
        raise ValueError("slots and slots4 differ in length")
    k4, v4 = _on(kq_pool, "kq_pool", "u8", page, at), _on(vq_pool, "vq_pool", "u8", page, at)
    if kq_pool.numel() != vq_pool.numel() or kq_pool.numel() % page:
        raise ValueError(f"4-bit pools of {kq_pool.numel()} and {vq_pool.numel()} bytes, expected the same multiple of {page}")
    return (_on(k_pool, "k_pool", "bf16", n, at), _on(v_pool, "v_pool", "bf16", n, at),
            _on(slots, "slots", "i32", 0, at, nullable=pages == 0), kq_pool.numel() // page, k4, v4,
            _on(slots4, "slots4", "i32", 0, at, nullable=pages == 0), pages)


def sa_kvq_pack(ctx, layout: Layout, k_pool, v_pool, slots, kq_pool, vq_pool, slots4, stream=None):
    """Quantises pages: slots[i] of the bf16 pools, every layer, into slots4[i] of the 4-bit pools (whose number of
    slots follows from their size).  slots, slots4: device int32."""
    k, v, s, n4, k4, v4, s4, pages = _convert_args(ctx, layout, k_pool, v_pool, slots, kq_pool, vq_pool, slots4)
    _check(load_library().sa_kvq_pack(_ctx_handle(ctx), ctypes.byref(layout), k, v, s, n4, k4, v4, s4, pages,
                                      _stream_of(ctx, stream)))


def sa_kvq_unpack(ctx, layout: Layout, kq_pool, vq_pool, slots4, k_pool, v_pool, slots, stream=None):
    """The way back: slots4[i] of the 4-bit pools, every layer, into slots[i] of the bf16 pools, exactly."""
    k, v, s, n4, k4, v4, s4, pages = _convert_args(ctx, layout, k_pool, v_pool, slots, kq_pool, vq_pool, slots4)
    _check(load_library().sa_kvq_unpack(_ctx_handle(ctx), ctypes.byref(layout), n4, k4, v4, s4, k, v, s, pages,
                                        _stream_of(ctx, stream)))


def sa_kvq_attn(ctx, layout: Layout, layer: int, q, kq_pool, vq_pool, q_len, kv_len, pages_indptr, pages_indices,
                softmax_scale: float, o, lse=None, causal: bool = True, stream=None):
    """Attention over a 4-bit cache: causal (as sa_segment_prefill_attn), or every query row over all keys of its
    sequence (causal=False; kv_len may be 0: rows of zeros, lse -inf)."""
    q_len, kv_len = _host_i32(q_len), _host_i32(kv_len)
    if q_len.shape != kv_len.shape:
        raise ValueError("q_len and kv_len differ in length")
    B, T, at = len(q_len), max(0, _total(q_len)), _device_of(ctx)
    n, rows = _kvq_bytes(layout, layout.num_slots), T * layout.num_q_heads
    _check(load_library().sa_kvq_attn(
        _ctx_handle(ctx), ctypes.byref(layout), int(layer), _on(q, "q", "bf16", rows * layout.head_dim, at, T == 0),
        _on(kq_pool, "kq_pool", "u8", n, at), _on(vq_pool, "vq_pool", "u8", n, at), B, _ptr(q_len), _ptr(kv_len),
        _table_on(pages_indptr, pages_indices, B, at, "page table",
                  pages_indices is None and not ((q_len > 0) & (kv_len > 0)).any()),
        int(bool(causal)), float(softmax_scale), _on(o, "o", "bf16", rows * layout.head_dim, at, T == 0),
        None if lse is None else _on(lse, "lse", "f32", rows, at), _stream_of(ctx, stream)))
