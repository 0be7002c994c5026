"""Codes of the operators of a layer of experts on the CPU: exported symbols, refusals of the encoders, verifier, dump, tensor
extents, what a launch refuses."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from paper_2603_24239_b200 import binding, experts
from tests import experts_oracle as orc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, SHAPE, UNSUPPORTED, SMALL, BAD_CODE, CUDA, TOO_LARGE = 0, -1, -2, -3, -4, -5, -6, -10
NAMES = ("routing", "quantize", "scaled_matmul", "combine")


def desc(name, **kw):
    d = {"routing": lambda: experts.RoutingDesc(tokens=10, experts=16, logits_stride=16, dtype=0, scoring=1, top_k=4, groups=4, top_groups=2, biased=1,
                                                masked=1, renormalise=1, factor=2.5),
         "quantize": lambda: experts.QuantizeDesc(rows=10, cols=272, out_rows=30, x_stride=272, codes_stride=272, scales_stride=3, dtype=1, gated=0,
                                                  copies=3, block_rows=1),
         "scaled_matmul": lambda: experts.ScaledMatmulDesc(rows=30, n=200, k=272, groups=5, x_stride=272, x_scales_stride=3, out_stride=200,
                                                           w_stride=(200 * 272, 272), out_dtype=1, grouped=1),
         "combine": lambda: experts.CombineDesc(tokens=10, top_k=3, rows=30, cols=200, y_stride=200, base_stride=200, out_stride=200, dtype=1, based=1)}[name]()
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def encode(name, cap=experts.CODE_BYTES, **kw):
    buf, size = (C.c_uint64 * (experts.CODE_BYTES // 8))(), C.c_size_t(0)
    st = getattr(binding.lib, "dvm_encode_" + name)(C.byref(desc(name, **kw)), buf, cap, C.byref(size))
    return st, buf, size.value


def test_library_exports_every_declared_symbol():
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dvm_experts.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(dvm_[a-z0-9_]+)\s*\(", hdr)) == set(experts.EXPORTS)
    sizes = {m[0]: int(m[1]) for m in re.findall(r"#define DVM_(\w+) (\d+)", hdr)}
    assert sizes == {"MAX_EXPERTS": experts.MAX_EXPERTS, "MAX_TOP_K": experts.MAX_TOP_K, "MAX_WEIGHT_GROUPS": experts.MAX_WEIGHT_GROUPS,
                     "SCALE_BLOCK": experts.SCALE_BLOCK, "EXPERTS_CODE_BYTES": experts.CODE_BYTES}


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (dict(tokens=0), OK), (dict(experts=512, logits_stride=512), OK), (dict(experts=513, logits_stride=513), TOO_LARGE), (dict(experts=0), INVALID),
    (dict(tokens=-1), INVALID), (dict(tokens=(1 << 23) + 1), TOO_LARGE), (dict(top_k=0), INVALID), (dict(top_k=8), OK), (dict(top_k=9), SHAPE),
    (dict(top_k=33, groups=1, top_groups=1), TOO_LARGE), (dict(groups=3), SHAPE), (dict(groups=0), INVALID), (dict(top_groups=5), SHAPE), (dict(top_groups=0), INVALID),
    (dict(groups=16, top_groups=4), OK), (dict(groups=64, top_groups=4, experts=64, logits_stride=64), TOO_LARGE), (dict(scoring=2), INVALID), (dict(dtype=2), INVALID),
    (dict(biased=2), INVALID), (dict(masked=-1), INVALID), (dict(factor=float("nan")), INVALID), (dict(factor=0.0), OK), (dict(logits_stride=-16), INVALID),
    (dict(logits_stride=0), OK)])
def test_routing_refusals(kw, want):
    assert encode("routing", **kw)[0] == want


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (dict(rows=0), OK), (dict(out_rows=0), OK), (dict(copies=0), SHAPE), (dict(copies=0, out_rows=10), OK), (dict(copies=33), TOO_LARGE), (dict(copies=-1), INVALID),
    (dict(cols=264), UNSUPPORTED), (dict(codes_stride=280), UNSUPPORTED), (dict(codes_stride=256), INVALID), (dict(codes_stride=288), OK), (dict(scales_stride=2), INVALID),
    (dict(x_stride=0), OK), (dict(x_stride=-272), INVALID), (dict(gated=1, x_stride=544), OK), (dict(gated=2), INVALID), (dict(dtype=3), INVALID), (dict(cols=0), INVALID),
    (dict(block_rows=128), INVALID), (dict(block_rows=128, copies=0, out_rows=10), OK), (dict(block_rows=128, copies=0, out_rows=10, gated=1), INVALID),
    (dict(block_rows=64, copies=0, out_rows=10), INVALID)])
def test_quantize_refusals(kw, want):
    assert encode("quantize", **kw)[0] == want


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (dict(rows=0), OK), (dict(k=264), UNSUPPORTED), (dict(x_stride=280), UNSUPPORTED), (dict(x_stride=0), UNSUPPORTED), (dict(rows=1, x_stride=0), OK),
    (dict(w_stride=(200 * 272, 280)), UNSUPPORTED), (dict(w_stride=(0, 272)), UNSUPPORTED), (dict(w_stride=(-16, 272)), INVALID), (dict(out_stride=199), INVALID),
    (dict(out_stride=203), OK), (dict(grouped=0), SHAPE), (dict(grouped=0, groups=1), OK), (dict(grouped=2), INVALID), (dict(groups=1024), OK), (dict(groups=1025), TOO_LARGE),
    (dict(groups=0), INVALID), (dict(n=0), INVALID), (dict(k=0), INVALID), (dict(out_dtype=2), INVALID), (dict(x_scales_stride=0), OK), (dict(x_scales_stride=-1), INVALID)])
def test_scaled_matmul_refusals(kw, want):
    assert encode("scaled_matmul", **kw)[0] == want


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (dict(tokens=0), OK), (dict(rows=0), OK), (dict(top_k=0), INVALID), (dict(top_k=33), TOO_LARGE), (dict(cols=0), INVALID), (dict(dtype=2), INVALID),
    (dict(based=2), INVALID), (dict(out_stride=100), INVALID), (dict(y_stride=0), OK), (dict(base_stride=-1), INVALID), (dict(based=0, base_stride=-1), OK), (dict(y_stride=-200), INVALID)])
def test_combine_refusals(kw, want):
    assert encode("combine", **kw)[0] == want


@pytest.mark.parametrize("name", NAMES)
def test_codes_verify_and_changed_ones_do_not(name):
    st, buf, size = encode(name)
    assert st == OK and binding.lib.dvm_verify(buf, size) == OK
    assert encode(name, cap=size - 4)[0] == SMALL
    enc = getattr(binding.lib, "dvm_encode_" + name)
    assert enc(None, buf, size, C.byref(C.c_size_t(0))) == INVALID and enc(C.byref(desc(name)), buf, size, None) == INVALID
    text = C.create_string_buffer(1 << 12)
    assert binding.lib.dvm_disassemble(buf, size, text, len(text)) == OK and b"kernel " + name.encode() in text.value
    assert binding.lib.dvm_disassemble(buf, size, text, 10) == SMALL
    assert binding.lib.dvm_verify(buf, size - 4) == BAD_CODE
    words = C.cast(buf, C.POINTER(C.c_uint32))
    nt = words[5] & 0xff
    for at, value in ((0, 7), (1, 11), (1, 3), (3, words[3] + 1), (4, words[4] + 1), (5, words[5] + 1), (5, words[5] ^ (1 << 24)),
                      (20 + 2 * nt, 0xffffffff), (20 + 2 * nt + 1, 0x80000000)):   # the last two: the descriptor's first size
        old, words[at] = words[at], value
        assert binding.lib.dvm_verify(buf, size) != OK, at
        words[at] = old
    assert binding.lib.dvm_verify(buf, size) == OK
    # neither the stacked launches nor dvm_run_host take these codes (refused before any CUDA call)
    ptrs = (C.c_void_p * nt)(*[256] * nt)
    tl = (C.POINTER(C.c_void_p) * 1)(C.cast(ptrs, C.POINTER(C.c_void_p)))
    args = (1, (C.c_void_p * 1)(C.addressof(buf)), (C.c_size_t * 1)(size), tl, (C.c_int * 1)(nt))
    assert binding.lib.dvm_launch_stacked(*args, None) == UNSUPPORTED
    assert binding.lib.dvm_launch_stacked_levels(*args, (C.c_int * 1)(0), None) == UNSUPPORTED
    assert binding.lib.dvm_launch_stacked_noalloc(*args, None) == UNSUPPORTED
    assert binding.lib.dvm_run_host(buf, size, ptrs, (C.c_size_t * nt)(*[64] * nt), nt, 256, 1 << 20, None) == UNSUPPORTED
    # a short tensor is refused by the checked launch, a missing one and a wrong count by every launch, before any CUDA call
    need = (C.c_int64 * nt)()
    assert binding.lib.dvm_tensor_extents(buf, size, need, nt) == OK
    for i in range(nt):
        if need[i]:
            have = [n - (k == i) for k, n in enumerate(need)]
            assert binding.lib.dvm_launch_checked(buf, size, ptrs, (C.c_size_t * nt)(*have), nt, None) == SMALL
            none = (C.c_void_p * nt)(*[None if k == i else 4096 * (k + 1) for k in range(nt)])
            assert binding.lib.dvm_launch(buf, size, none, nt, None) == INVALID
    assert binding.lib.dvm_launch(buf, size, ptrs, nt - 1, None) == INVALID


def test_extents():
    def of(name, **kw):
        st, buf, size = encode(name, **kw)
        assert st == OK
        return dvm.tensor_extents(binding.Code(buf, size, []))
    assert of("routing") == [10 * 16 * 4, 64, 40, 160, 160, 160, 68, 0]
    assert of("routing", biased=0, masked=0, dtype=1, logits_stride=20) == [2 * (9 * 20 + 16), 160, 160, 160, 68, 0]
    assert of("routing", tokens=128)[-1] == 0 and of("routing", tokens=129)[-1] == 9 * 16 and of("routing", tokens=16 * 592 + 1, experts=18, logits_stride=18, groups=1, top_groups=1)[-1] == 297 * 32
    assert of("quantize") == [10 * 272 * 2, 120, 30 * 272, 30 * 3 * 4]
    assert of("quantize", gated=1, x_stride=600) == [2 * (9 * 600 + 544), 120, 30 * 272, 30 * 3 * 4]
    assert of("quantize", copies=0, rows=300, out_rows=300, block_rows=128, dtype=0) == [300 * 272 * 4, 300 * 272, 3 * 3 * 4]
    assert of("quantize", rows=0) == [0] * 4
    assert of("scaled_matmul")[:6] == [30 * 272, 30 * 12, 5 * 200 * 272, 5 * 2 * 3 * 4, 24, 30 * 200 * 2]
    assert of("scaled_matmul", rows=0) == [0] * 7
    assert of("scaled_matmul", grouped=0, groups=1, out_dtype=0)[4] == 30 * 200 * 4
    assert of("combine") == [30 * 400, 120, 120, 10 * 400, 10 * 400]
    assert of("combine", based=0, dtype=0, out_stride=210) == [30 * 800, 120, 120, 4 * (9 * 210 + 200)]


def test_binding_checks_tensors():
    b16, f8, i32 = torch.bfloat16, torch.float8_e4m3fn, torch.int32
    x, codes, scales = torch.zeros(4, 256, dtype=b16), torch.zeros(12, 256, dtype=f8), torch.zeros(12, 2)
    places = torch.zeros(4, 3, dtype=i32)
    assert dvm.verify(dvm.encode_routing(x, 4)) == 0
    for bad in (dict(logits=x.double()), dict(logits=x.t()), dict(logits=x[0]), dict(scoring="top"), dict(top_k=0), dict(groups=3)):
        with pytest.raises(dvm.DvmError):
            dvm.encode_routing(**{**dict(logits=x, top_k=4), **bad})
    good = dict(x=x, codes=codes, scales=scales, places=places)
    assert dvm.verify(dvm.encode_quantize(**good)) == 0 and dvm.verify(dvm.encode_quantize(**{**good, "codes": codes.view(torch.uint8)})) == 0
    for bad in (dict(x=x.half()), dict(codes=codes.float()), dict(scales=scales.double()), dict(scales=scales[:, :1]), dict(places=places.long()), dict(places=places[:3]),
                dict(places=places[:, :0]), dict(places=None), dict(gated=True), dict(block_rows=128), dict(block_rows=2), dict(x=x[:, ::2], codes=codes[:, :128], scales=scales[:, :1])):
        with pytest.raises(dvm.DvmError):
            dvm.encode_quantize(**{**good, **bad})
    w, ws, out, starts = torch.zeros(5, 200, 256, dtype=f8), torch.zeros(5, 2, 2), torch.zeros(12, 200), torch.zeros(6, dtype=i32)
    good = dict(x=codes, x_scales=scales, w=w, w_scales=ws, out=out, starts=starts)
    assert dvm.verify(dvm.encode_scaled_matmul(**good)) == 0
    for bad in (dict(x=codes.float()), dict(x=codes[:, :128]), dict(x_scales=scales[:11]), dict(w=w[:, :, ::2]), dict(w=w[0]), dict(w_scales=ws.transpose(1, 2)), dict(w_scales=ws[:4]),
                dict(out=out[:, :100]), dict(out=out.half()), dict(starts=starts[:5]), dict(starts=starts.long()), dict(starts=None)):
        with pytest.raises(dvm.DvmError):
            dvm.encode_scaled_matmul(**{**good, **bad})
    y, weights = torch.zeros(12, 200), torch.zeros(4, 3)
    good = dict(y=y, places=places, weights=weights, out=out[:4], base=out[4:8])
    assert dvm.verify(dvm.encode_combine(**good)) == 0
    for bad in (dict(y=y.to(b16)), dict(places=places[0]), dict(places=places.long()), dict(weights=weights.double()), dict(weights=weights[:, :2]), dict(out=out[:3]), dict(base=out),
                dict(base=out[:4].to(b16)), dict(y=y.double())):
        with pytest.raises(dvm.DvmError):
            dvm.encode_combine(**{**good, **bad})


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: only for a machine that cannot launch")
def test_what_a_launch_refuses():
    """A refusal, or on a machine without a device its CUDA error."""
    far = [0x100000 * (i + 1) for i in range(16)]

    def launched(name, places=(), **kw):
        st, buf, size = encode(name, **kw)
        assert st == OK
        nt = C.cast(buf, C.POINTER(C.c_uint32))[5] & 0xff
        at = list(far[:nt])
        for i, p in places:
            at[i] = p
        return binding.lib.dvm_launch(buf, size, (C.c_void_p * nt)(*at), nt, None)
    for name in NAMES:
        assert launched(name) == CUDA, name
    # outputs that begin where another tensor does
    assert launched("routing", [(3, far[2])]) == INVALID and launched("routing", [(5, far[4])]) == INVALID and launched("routing", [(1, far[0])]) == CUDA
    assert launched("quantize", [(2, far[0])]) == INVALID and launched("quantize", [(3, far[2])]) == INVALID
    assert launched("scaled_matmul", [(5, far[1])]) == INVALID and launched("scaled_matmul", [(6, far[5])]) == INVALID and launched("scaled_matmul", [(2, far[0])]) == CUDA
    assert launched("combine", [(4, far[0])]) == INVALID and launched("combine", [(4, far[3])]) == CUDA and launched("combine", [(4, far[3])], out_stride=208) == INVALID
    # alignment: elements everywhere, 16 bytes for codes and the workspace
    for i in (0, 1, 2, 3, 4, 5, 6):
        assert launched("routing", [(i, far[i] + 2)]) == INVALID, i
    assert launched("quantize", [(0, far[0] + 2)]) == CUDA and launched("quantize", [(0, far[0] + 1)]) == INVALID and launched("quantize", [(2, far[2] + 8)]) == INVALID
    assert launched("scaled_matmul", [(0, far[0] + 8)]) == INVALID and launched("scaled_matmul", [(2, far[2] + 8)]) == INVALID and launched("scaled_matmul", [(6, far[6] + 8)]) == INVALID
    assert launched("scaled_matmul", [(5, far[5] + 2)]) == CUDA and launched("scaled_matmul", [(5, far[5] + 2)], out_dtype=0) == INVALID
    assert launched("combine", [(0, far[0] + 2)]) == CUDA and launched("combine", [(0, far[0] + 1)]) == INVALID


def test_oracle_codes_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(orc.decode(codes), want, equal_nan=True)
    r = np.random.default_rng(0)
    v = np.concatenate([r.standard_normal(4000).astype(np.float32).astype(np.float64) * 2.0 ** r.integers(-12, 8, 4000), want[np.isfinite(want)]])
    v = np.clip(v, -448, 448)
    # every border between two codes goes to the even one
    t = orc.e4m3_values()
    v = np.concatenate([v, (t[1:] + t[:-1]) / 2])
    got = torch.from_numpy(v).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(orc.encode(v), got)
