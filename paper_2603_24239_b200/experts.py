"""ctypes binding of include/dvm_experts.h: the codes of the operators of a layer of experts.

As in `serving`, the encode functions read sizes, strides and element types from the tensors an instance will be launched
with and return a Code; `launch(code, tensors, stream)` runs it on those or any others of the same layout.  Codes of 8-bit
values are tensors of float8_e4m3fn (or uint8, the same bytes).
"""
from __future__ import annotations

import ctypes as C

from .binding import Code, DvmError, _check, lib
from .serving import _adjacent, _dtype, _like, _same

_i64, _i32 = C.c_int64, C.c_int32
CODE_BYTES = 512   # DVM_EXPERTS_CODE_BYTES
MAX_EXPERTS, MAX_TOP_K, MAX_WEIGHT_GROUPS, SCALE_BLOCK = 512, 32, 1024, 128
SCORING = {"softmax": 0, "sigmoid": 1}


class RoutingDesc(C.Structure):
    _fields_ = ([(n, _i64) for n in ("tokens", "experts", "logits_stride")]
                + [(n, _i32) for n in ("dtype", "scoring", "top_k", "groups", "top_groups", "biased", "masked", "renormalise")] + [("factor", C.c_float)])


class QuantizeDesc(C.Structure):
    _fields_ = ([(n, _i64) for n in ("rows", "cols", "out_rows", "x_stride", "codes_stride", "scales_stride")]
                + [(n, _i32) for n in ("dtype", "gated", "copies", "block_rows")])


class ScaledMatmulDesc(C.Structure):
    _fields_ = ([(n, _i64) for n in ("rows", "n", "k", "groups", "x_stride", "x_scales_stride", "out_stride")] + [("w_stride", _i64 * 2)]
                + [(n, _i32) for n in ("out_dtype", "grouped")])


class CombineDesc(C.Structure):
    _fields_ = ([(n, _i64) for n in ("tokens", "top_k", "rows", "cols", "y_stride", "base_stride", "out_stride")]
                + [(n, _i32) for n in ("dtype", "based")])


_sig = {
    "dvm_encode_routing": ([C.POINTER(RoutingDesc), C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)], C.c_int),
    "dvm_encode_quantize": ([C.POINTER(QuantizeDesc), C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)], C.c_int),
    "dvm_encode_scaled_matmul": ([C.POINTER(ScaledMatmulDesc), C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)], C.c_int),
    "dvm_encode_combine": ([C.POINTER(CombineDesc), C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)], C.c_int),
    "dvm_last_scaled_matmul_tile": ([C.POINTER(C.c_int)], C.c_int),
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


def _blocks(n: int) -> int:
    return -(-n // SCALE_BLOCK)


def _is_codes(t, what: str):
    import torch
    if t.dtype not in (torch.float8_e4m3fn, torch.uint8):
        raise DvmError(-1, f"{what} are {t.dtype}: float8_e4m3fn (or its bytes, uint8) is wanted")


def _is(t, what: str, dtype, shape, dense: bool = True):
    if t.dtype != dtype or (dense and not t.is_contiguous()):
        raise DvmError(-1, f"{what}: a {'dense ' if dense else ''}tensor of {dtype} is wanted")
    _like(t, what, shape)


def encode_routing(logits, top_k: int, scoring: str = "softmax", biased: bool = False, groups: int = 1, top_groups: int = 1,
                   renormalise: bool = False, factor: float = 1.0, masked: bool = False) -> Code:
    """dvm_encode_routing for logits [tokens, experts].  Launch with (logits[, bias][, positions], ids, weights, places, starts,
    workspace): bias [experts] fp32, positions [tokens] int32 (negative: the token takes no part); ids, places int32 and weights
    fp32 [tokens, top_k], starts [experts + 1] int32, the workspace tensor_extents(code)[-1] bytes (0: any tensor)."""
    _adjacent(logits, "logits", 2)
    if scoring not in SCORING:
        raise DvmError(-1, f"scoring is {scoring!r}: softmax or sigmoid is wanted")
    t, e = logits.shape
    d = RoutingDesc(t, e, logits.stride(0), _dtype(logits, "logits"), SCORING[scoring], top_k, groups, top_groups, int(bool(biased)),
                    int(bool(masked)), int(bool(renormalise)), factor)
    return _code(lib.dvm_encode_routing, d, [(t, top_k), (t, top_k), (t, top_k), (e + 1,)])


def encode_quantize(x, codes, scales, places=None, gated: bool = False, block_rows: int = 1) -> Code:
    """dvm_encode_quantize for x [rows, cols] (`gated`: [rows, 2 cols], gate and up columns), codes [out_rows, cols], scales
    [out_rows / block_rows, cols / 128] (rounded up) fp32.  With places [rows, copies] int32 row t goes to those rows of the codes.
    Launch with (x[, places], codes, scales)."""
    import torch
    _adjacent(x, "x", 2)
    _adjacent(codes, "codes", 2)
    _is_codes(codes, "codes")
    _adjacent(scales, "scales", 2)
    rows, out_rows, cols, copies = x.shape[0], codes.shape[0], codes.shape[1], 0
    _like(x, "x", (rows, cols * (2 if gated else 1)))
    if places is not None:
        copies = places.shape[1] if places.dim() == 2 else 0
        _is(places, "places", torch.int32, (rows, copies))
        if copies == 0:
            raise DvmError(-2, "places has no column")
    if block_rows not in (1, SCALE_BLOCK):
        raise DvmError(-1, f"block_rows is {block_rows}: 1 or {SCALE_BLOCK} is wanted")
    _is(scales, "scales", torch.float32, (-(-out_rows // block_rows), _blocks(cols)), dense=False)
    d = QuantizeDesc(rows, cols, out_rows, x.stride(0), codes.stride(0), scales.stride(0), _dtype(x, "x"), int(bool(gated)), copies, block_rows)
    return _code(lib.dvm_encode_quantize, d, [(out_rows, cols), tuple(scales.shape)])


def encode_scaled_matmul(x, x_scales, w, w_scales, out, starts=None) -> Code:
    """dvm_encode_scaled_matmul for codes x [rows, k] with x_scales [rows, k / 128], codes w [groups, n, k] with w_scales [groups,
    n / 128, k / 128] (all rounded up, fp32, the latter dense) and out [rows, n].  With starts [groups + 1] int32 the rows
    starts[g] <= r < starts[g + 1] meet w[g]; without, groups is 1.
    Launch with (x, x_scales, w, w_scales[, starts], out, workspace); the workspace has tensor_extents(code)[-1] bytes (0: any
    tensor) and belongs to one launch at a time."""
    import torch
    _adjacent(x, "x", 2)
    _is_codes(x, "x")
    _adjacent(w, "w", 3)
    _is_codes(w, "w")
    rows, k = x.shape
    groups, n, _ = w.shape
    _like(w, "w", (groups, n, k))
    _adjacent(x_scales, "x_scales", 2)
    _is(x_scales, "x_scales", torch.float32, (rows, _blocks(k)), dense=False)
    _is(w_scales, "w_scales", torch.float32, (groups, _blocks(n), _blocks(k)))
    _adjacent(out, "out", 2)
    _like(out, "out", (rows, n))
    if starts is not None:
        _is(starts, "starts", torch.int32, (groups + 1,))
    d = ScaledMatmulDesc(rows, n, k, groups, x.stride(0), x_scales.stride(0), out.stride(0), tuple(w.stride()[:2]), _dtype(out, "out"),
                         int(starts is not None))
    return _code(lib.dvm_encode_scaled_matmul, d, [(rows, n)])


def encode_combine(y, places, weights, out, base=None) -> Code:
    """dvm_encode_combine for y [rows, cols], places int32 and weights fp32 [tokens, top_k], out and base [tokens, cols].
    Launch with (y, places, weights[, base], out); out may be base."""
    import torch
    _adjacent(y, "y", 2)
    _adjacent(out, "out", 2)
    if places.dim() != 2:
        raise DvmError(-1, "places is a matrix [tokens, top_k]")
    tokens, top_k = places.shape
    rows, cols = y.shape
    _is(places, "places", torch.int32, (tokens, top_k))
    _is(weights, "weights", torch.float32, (tokens, top_k))
    _like(out, "out", (tokens, cols))
    dtype = _same(_dtype(y, "y"), _dtype(out, "out"), "y and out")
    if base is not None:
        _adjacent(base, "base", 2)
        _like(base, "base", (tokens, cols))
        _same(dtype, _dtype(base, "base"), "y and base")
    d = CombineDesc(tokens, top_k, rows, cols, y.stride(0), base.stride(0) if base is not None else 0, out.stride(0), dtype, int(base is not None))
    return _code(lib.dvm_encode_combine, d, [(tokens, cols)])


def last_scaled_matmul_tile() -> int:
    """dvm_last_scaled_matmul_tile: rows of the tiles that this thread's last scaled product worked on."""
    out = C.c_int(-1)
    _check(lib.dvm_last_scaled_matmul_tile(C.byref(out)), "dvm_last_scaled_matmul_tile")
    return out.value
