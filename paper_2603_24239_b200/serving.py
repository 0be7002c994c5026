"""ctypes binding of include/dvm_serving.h: the codes of a serving step's operators.

The encode functions read sizes, strides and element types from the tensors an instance will be launched with and
return a Code; `launch(code, tensors, stream)` runs it on those or any others of the same layout.  As elsewhere in the
binding, a launch passes device addresses: the caller keeps the tensors alive until the stream has run it.
"""
from __future__ import annotations

import ctypes as C

from .binding import BF16, F32, Code, DvmError, _check, lib

_i64, _i32 = C.c_int64, C.c_int32
CODE_BYTES = 512   # DVM_SERVING_CODE_BYTES
MAX_REQUESTS = 8192


class PagingDesc(C.Structure):
    _fields_ = [(n, _i64) for n in ("requests", "max_blocks", "page_size", "rows", "free_pages")]


class RotaryDesc(C.Structure):
    _fields_ = ([(n, _i64) for n in ("tokens", "q_heads", "kv_heads", "head_dim", "rotary_dim", "angle_rows", "pages", "page_size")]
                + [(n, _i64 * 2) for n in ("q_stride", "k_stride", "v_stride", "q_out_stride", "k_out_stride")]
                + [(n, _i64 * 3) for n in ("k_cache_stride", "v_cache_stride")]
                + [(n, _i32) for n in ("dtype", "weight_dtype", "out_dtype", "norm", "interleaved", "paged")] + [("eps", C.c_float)])


class AttentionDesc(C.Structure):
    _fields_ = ([(n, _i64) for n in ("requests", "rows", "q_heads", "kv_heads", "head_dim", "pages", "page_size", "max_blocks", "window",
                                     "sinks", "max_q")]
                + [(n, _i64 * 2) for n in ("q_stride", "out_stride")] + [(n, _i64 * 3) for n in ("k_stride", "v_stride")]
                + [(n, _i32) for n in ("dtype", "out_dtype")] + [("scale", C.c_float)])


_sig = {
    "dvm_encode_paging": ([C.POINTER(PagingDesc), C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)], C.c_int),
    "dvm_encode_rotary": ([C.POINTER(RotaryDesc), C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)], C.c_int),
    "dvm_encode_attention": ([C.POINTER(AttentionDesc), C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)], C.c_int),
    "dvm_last_attention_kernel": ([C.POINTER(C.c_int)], C.c_int),
}
for _name, (_args, _res) in _sig.items():
    _f = getattr(lib, _name)
    _f.argtypes = _args
    _f.restype = _res
EXPORTS = tuple(_sig)


def _code(fn, desc, out_shapes) -> Code:
    buf, size = (C.c_uint64 * (CODE_BYTES // 8))(), C.c_size_t(0)
    _check(fn(C.byref(desc), buf, CODE_BYTES, C.byref(size)), fn.__name__)
    return Code(buf, size.value, out_shapes)


def _dtype(t, what: str) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise DvmError(-1, f"{what} is {t.dtype}: bf16 or fp32 is wanted")


def _adjacent(t, what: str, rank: int):
    if t.dim() != rank:
        raise DvmError(-1, f"{what} has {t.dim()} dimensions: {rank} are wanted")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise DvmError(-1, f"the last dimension of {what} is not adjacent")


def _like(t, what: str, shape):
    if tuple(t.shape) != tuple(shape):
        raise DvmError(-2, f"{what} is {tuple(t.shape)}: {tuple(shape)} is wanted")


def _same(a: int, b: int, what: str) -> int:
    if a != b:
        raise DvmError(-1, f"the element types of {what} differ")
    return a


def encode_paging(requests: int, max_blocks: int, page_size: int, rows: int, free_pages: int) -> Code:
    """dvm_encode_paging.  Launch with (cached, fresh, free, table, starts, lengths, positions, slots, taken), all int32:
    from the cached and new tokens of every request, the new tokens' rows, positions and cache slots; the blocks they open
    take pages from `free` and are written into `table`."""
    return _code(lib.dvm_encode_paging, PagingDesc(requests, max_blocks, page_size, rows, free_pages),
                 [(requests, max_blocks), (requests + 1,), (requests,), (rows,), (rows,), (1,)])


def encode_rotary(q, k, angles, q_out, v=None, wq=None, wk=None, k_out=None, k_cache=None, v_cache=None, eps: float = 1e-6,
                  interleaved: bool = False) -> Code:
    """dvm_encode_rotary for tensors of these layouts: q [tokens, q_heads, dim], k and v [tokens, kv_heads, dim], weights wq
    and wk [dim] (both or neither: no norm), angles [rows, rotary_dim] fp32 = [cos | sin].  With k_cache and v_cache
    [pages, page_size, kv_heads, dim] keys and values go to the cache, else keys go to k_out [tokens, kv_heads, dim].
    Launch with (q, k[, v][, wq, wk], angles, positions[, slots], q_out, k_cache, v_cache) or (..., q_out, k_out)."""
    import torch
    d = RotaryDesc()
    paged = k_cache is not None
    if paged != (v_cache is not None) or paged != (v is not None) or paged == (k_out is not None) or (wq is None) != (wk is None):
        raise DvmError(-1, "encode_rotary: either v, k_cache and v_cache or k_out; both weights or none")
    _adjacent(q, "q", 3)
    t, hq, dim = q.shape
    _adjacent(k, "k", 3)
    hk = k.shape[1]
    _like(k, "k", (t, hk, dim))
    _adjacent(q_out, "q_out", 3)
    _like(q_out, "q_out", (t, hq, dim))
    if angles.dim() != 2 or angles.dtype != torch.float32 or not angles.is_contiguous():
        raise DvmError(-1, "angles is a dense fp32 table [positions, rotary_dim]")
    d.tokens, d.q_heads, d.kv_heads, d.head_dim, d.rotary_dim, d.angle_rows = t, hq, hk, dim, angles.shape[1], angles.shape[0]
    d.dtype = _same(_dtype(q, "q"), _dtype(k, "k"), "q and k")
    d.out_dtype = _dtype(q_out, "q_out")
    d.q_stride[:], d.k_stride[:], d.q_out_stride[:] = q.stride()[:2], k.stride()[:2], q_out.stride()[:2]
    outs = [(t, hq, dim)]
    if paged:
        _adjacent(v, "v", 3)
        _like(v, "v", (t, hk, dim))
        _same(d.dtype, _dtype(v, "v"), "q and v")
        for c, what in ((k_cache, "k_cache"), (v_cache, "v_cache")):
            _adjacent(c, what, 4)
            _like(c, what, (k_cache.shape[0], k_cache.shape[1], hk, dim))
            _same(d.out_dtype, _dtype(c, what), f"q_out and {what}")
        d.paged, d.pages, d.page_size = 1, k_cache.shape[0], k_cache.shape[1]
        d.v_stride[:], d.k_cache_stride[:], d.v_cache_stride[:] = v.stride()[:2], k_cache.stride()[:3], v_cache.stride()[:3]
        outs += [tuple(k_cache.shape), tuple(v_cache.shape)]
    else:
        _adjacent(k_out, "k_out", 3)
        _like(k_out, "k_out", (t, hk, dim))
        _same(d.out_dtype, _dtype(k_out, "k_out"), "q_out and k_out")
        d.k_out_stride[:] = k_out.stride()[:2]
        outs.append((t, hk, dim))
    if wq is not None:
        for w, what in ((wq, "wq"), (wk, "wk")):
            _adjacent(w, what, 1)
            _like(w, what, (dim,))
        d.norm, d.eps, d.weight_dtype = 1, eps, _same(_dtype(wq, "wq"), _dtype(wk, "wk"), "wq and wk")
    d.interleaved = int(bool(interleaved))
    return _code(lib.dvm_encode_rotary, d, outs)


def encode_attention(q, k_cache, v_cache, table, out, scale: float, window: int = 0, sinks: int = 0, max_q: int | None = None) -> Code:
    """dvm_encode_attention for tensors of these layouts: q and out [rows, q_heads, dim], caches [pages, page_size, kv_heads,
    dim], table [requests, max_blocks] int32.  max_q: most query rows of one request (default: all rows); 1 takes the
    kernel for single tokens.  Launch with (q, k_cache, v_cache, table, starts, lengths, out, workspace); the workspace has
    tensor_extents(code)[-1] bytes (0: any tensor) and belongs to one launch at a time."""
    import torch
    d = AttentionDesc()
    _adjacent(q, "q", 3)
    rows, hq, dim = q.shape
    _adjacent(out, "out", 3)
    _like(out, "out", (rows, hq, dim))
    _adjacent(k_cache, "k_cache", 4)
    pages, page_size, hk, _ = k_cache.shape
    _like(k_cache, "k_cache", (pages, page_size, hk, dim))
    _adjacent(v_cache, "v_cache", 4)
    _like(v_cache, "v_cache", (pages, page_size, hk, dim))
    if table.dim() != 2 or table.dtype != torch.int32 or not table.is_contiguous():
        raise DvmError(-1, "table is a dense int32 matrix [requests, max_blocks]")
    d.requests, d.max_blocks = table.shape
    d.rows, d.q_heads, d.kv_heads, d.head_dim, d.pages, d.page_size = rows, hq, hk, dim, pages, page_size
    d.window, d.sinks, d.max_q, d.scale = window, sinks, max(rows, 1) if max_q is None else max_q, scale
    d.q_stride[:], d.out_stride[:], d.k_stride[:], d.v_stride[:] = q.stride()[:2], out.stride()[:2], k_cache.stride()[:3], v_cache.stride()[:3]
    d.dtype = _same(_same(_dtype(q, "q"), _dtype(k_cache, "k_cache"), "q and k_cache"), _dtype(v_cache, "v_cache"), "q and v_cache")
    d.out_dtype = _dtype(out, "out")
    return _code(lib.dvm_encode_attention, d, [(rows, hq, dim)])


def last_attention_kernel() -> str:
    """dvm_last_attention_kernel: which kernel this thread's last attention launch ran on."""
    out = C.c_int(-1)
    _check(lib.dvm_last_attention_kernel(C.byref(out)), "dvm_last_attention_kernel")
    return ("plain", "single", "prompt")[out.value]
