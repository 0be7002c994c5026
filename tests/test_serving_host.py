"""Serving codes on the CPU: exported symbols, refusals of the encoders, verifier, dump, tensor extents."""
import ctypes as C
import os
import re

import pytest
import torch

import paper_2603_24239_b200 as dvm
from paper_2603_24239_b200 import binding, serving

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, SHAPE, UNSUPPORTED, SMALL, BAD_CODE, TOO_LARGE = 0, -1, -2, -3, -4, -5, -10


def _encode(fn, d, cap=serving.CODE_BYTES):
    buf, size = (C.c_uint64 * (serving.CODE_BYTES // 8))(), C.c_size_t(0)
    return fn(C.byref(d), buf, cap, C.byref(size)), buf, size.value


def paging(**kw):
    d = serving.PagingDesc(5, 7, 16, 100, 9)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def rotary(**kw):
    d = serving.RotaryDesc(tokens=10, q_heads=4, kv_heads=2, head_dim=64, rotary_dim=64, angle_rows=50, pages=3, page_size=16,
                           q_stride=(256, 64), k_stride=(128, 64), v_stride=(128, 64), q_out_stride=(256, 64),
                           k_cache_stride=(2048, 128, 64), v_cache_stride=(2048, 128, 64), dtype=1, weight_dtype=1, out_dtype=1, norm=1,
                           paged=1, eps=1e-6)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def attention(**kw):
    d = serving.AttentionDesc(requests=3, rows=20, q_heads=8, kv_heads=2, head_dim=64, pages=11, page_size=16, max_blocks=4, max_q=20,
                              q_stride=(512, 64), out_stride=(512, 64), k_stride=(2048, 128, 64), v_stride=(2048, 128, 64), dtype=1,
                              out_dtype=1, scale=0.125)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_library_exports_every_declared_symbol():
    hdr = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "dvm_serving.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(dvm_[a-z0-9_]+)\s*\(", hdr)) == set(serving.EXPORTS)
    sizes = {m[0]: int(m[1]) for m in re.findall(r"#define (DVM_MAX_REQUESTS|DVM_SERVING_CODE_BYTES) (\d+)", hdr)}
    assert sizes == {"DVM_MAX_REQUESTS": serving.MAX_REQUESTS, "DVM_SERVING_CODE_BYTES": serving.CODE_BYTES}


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (dict(requests=0), OK), (dict(rows=0), OK), (dict(free_pages=0, max_blocks=0), OK), (dict(page_size=1), OK),
    (dict(requests=8192), OK), (dict(requests=8193), TOO_LARGE), (dict(requests=-1), INVALID), (dict(page_size=0), INVALID),
    (dict(rows=-1), INVALID), (dict(rows=1 << 31), INVALID), (dict(free_pages=-1), INVALID), (dict(max_blocks=-2), INVALID)])
def test_paging_refusals(kw, want):
    assert _encode(binding.lib.dvm_encode_paging, paging(**kw))[0] == want


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (dict(tokens=0), OK), (dict(rotary_dim=0), OK), (dict(rotary_dim=32), OK), (dict(norm=0, weight_dtype=9), OK),
    (dict(head_dim=60, rotary_dim=56), UNSUPPORTED), (dict(rotary_dim=36), UNSUPPORTED), (dict(rotary_dim=72), INVALID),
    (dict(head_dim=264, rotary_dim=64), UNSUPPORTED), (dict(dtype=2), INVALID), (dict(out_dtype=3), INVALID), (dict(weight_dtype=2), INVALID),
    (dict(norm=2), INVALID), (dict(interleaved=-1), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(q_stride=(-256, 64)), INVALID), (dict(q_stride=(0, 64)), OK), (dict(q_out_stride=(0, 64)), INVALID),
    (dict(q_out_stride=(64, 64)), INVALID), (dict(q_out_stride=(64, 640)), OK), (dict(k_cache_stride=(2048, 64, 64)), INVALID),
    (dict(k_cache_stride=(2048, 64, 1024)), OK), (dict(v_cache_stride=(1024, 128, 64)), INVALID), (dict(page_size=0), INVALID),
    (dict(pages=1 << 30), INVALID), (dict(q_stride=(1 << 50, 64)), INVALID), (dict(q_heads=65536), TOO_LARGE),
    (dict(paged=0, k_out_stride=(128, 64)), OK), (dict(paged=0, k_out_stride=(64, 64)), INVALID)])
def test_rotary_refusals(kw, want):
    assert _encode(binding.lib.dvm_encode_rotary, rotary(**kw))[0] == want


@pytest.mark.parametrize("kw,want", [
    ({}, OK), (dict(rows=0), OK), (dict(requests=0), OK), (dict(pages=0), OK), (dict(head_dim=63), OK), (dict(window=5, sinks=3), OK),
    (dict(q_heads=7), SHAPE), (dict(kv_heads=0), INVALID), (dict(head_dim=257), UNSUPPORTED), (dict(page_size=24), UNSUPPORTED),
    (dict(page_size=4), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(window=-1), INVALID), (dict(sinks=-1), INVALID), (dict(max_q=0), INVALID), (dict(dtype=2), INVALID), (dict(out_dtype=2), INVALID),
    (dict(out_stride=(512, 32)), INVALID), (dict(out_stride=(0, 64)), INVALID), (dict(q_stride=(0, 0)), OK), (dict(k_stride=(0, 0, 0)), OK),
    (dict(k_stride=(-1, 128, 64)), INVALID), (dict(requests=8193), TOO_LARGE), (dict(kv_heads=1, q_heads=129), UNSUPPORTED),
    (dict(max_blocks=1 << 28), UNSUPPORTED)])
def test_attention_refusals(kw, want):
    assert _encode(binding.lib.dvm_encode_attention, attention(**kw))[0] == want


@pytest.mark.parametrize("fn,desc", [("dvm_encode_paging", paging), ("dvm_encode_rotary", rotary), ("dvm_encode_attention", attention)])
def test_codes_verify_and_changed_ones_do_not(fn, desc):
    enc = getattr(binding.lib, fn)
    st, buf, size = _encode(enc, desc())
    assert st == OK and binding.lib.dvm_verify(buf, size) == OK
    assert _encode(enc, desc(), cap=size - 4)[0] == SMALL
    assert enc(None, buf, size, C.byref(C.c_size_t(0))) == INVALID
    text = C.create_string_buffer(1 << 12)
    assert binding.lib.dvm_disassemble(buf, size, text, len(text)) == OK and fn.split("_")[-1].encode() in text.value
    assert binding.lib.dvm_disassemble(buf, size, text, 10) == SMALL
    assert binding.lib.dvm_verify(buf, size - 4) == BAD_CODE
    words = C.cast(buf, C.POINTER(C.c_uint32))
    nt = words[5] & 0xff
    for at, value in ((0, 7), (1, 9), (3, words[3] + 1), (4, words[4] + 1), (5, words[5] + 1), (5, words[5] ^ (1 << 24)),
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
    # a short tensor is refused by the checked launch, also before any CUDA call
    need = (C.c_int64 * nt)()
    assert binding.lib.dvm_tensor_extents(buf, size, need, nt) == OK
    for i in range(nt):
        if need[i]:
            have = [n - (k == i) for k, n in enumerate(need)]
            assert binding.lib.dvm_launch_checked(buf, size, ptrs, (C.c_size_t * nt)(*have), nt, None) == SMALL


def test_extents():
    st, buf, size = _encode(binding.lib.dvm_encode_paging, paging())
    c = binding.Code(buf, size, [])
    assert dvm.tensor_extents(c) == [20, 20, 36, 140, 24, 20, 400, 400, 4]
    st, buf, size = _encode(binding.lib.dvm_encode_rotary, rotary(q_stride=(300, 70)))
    assert dvm.tensor_extents(binding.Code(buf, size, [])) == [
        2 * (9 * 300 + 3 * 70 + 64), 2 * 10 * 128, 2 * 10 * 128, 128, 128, 50 * 64 * 4, 40, 40, 2 * 10 * 256, 2 * 3 * 2048, 2 * 3 * 2048]
    st, buf, size = _encode(binding.lib.dvm_encode_rotary, rotary(paged=0, norm=0, out_dtype=0, k_out_stride=(128, 64)))
    assert dvm.tensor_extents(binding.Code(buf, size, [])) == [2 * 10 * 256, 2 * 10 * 128, 50 * 64 * 4, 40, 4 * 10 * 256, 4 * 10 * 128]
    st, buf, size = _encode(binding.lib.dvm_encode_attention, attention())
    assert dvm.tensor_extents(binding.Code(buf, size, [])) == [2 * 20 * 512, 2 * 11 * 2048, 2 * 11 * 2048, 48, 16, 12, 2 * 20 * 512, 0]
    st, buf, size = _encode(binding.lib.dvm_encode_attention, attention(max_q=1))
    assert dvm.tensor_extents(binding.Code(buf, size, []))[-1] == 296 * (16 + 2 * 4 * (64 + 2) * 4)
    st, buf, size = _encode(binding.lib.dvm_encode_attention, attention(rows=0))
    assert dvm.tensor_extents(binding.Code(buf, size, [])) == [0] * 8


def test_binding_checks_tensors():
    b16 = torch.bfloat16
    q, k, cache = torch.zeros(4, 8, 64, dtype=b16), torch.zeros(4, 2, 64, dtype=b16), torch.zeros(3, 16, 2, 64, dtype=b16)
    ang, table = torch.zeros(9, 64), torch.zeros(2, 3, dtype=torch.int32)
    good = dict(q=q, k_cache=cache, v_cache=cache.clone(), table=table, out=torch.zeros_like(q), scale=1.0)
    assert dvm.verify(dvm.encode_attention(**good)) == 0
    for change in (dict(table=table.long()), dict(table=table.t()), dict(out=torch.zeros(4, 8, 32, dtype=b16)), dict(q=q.float()),
                   dict(q=q.half()), dict(v_cache=cache[:2]), dict(k_cache=cache.transpose(2, 3)), dict(q=q[0])):
        with pytest.raises(dvm.DvmError):
            dvm.encode_attention(**{**good, **change})
    good = dict(q=q, k=k, v=k.clone(), angles=ang, q_out=q, k_cache=cache, v_cache=cache)
    assert dvm.verify(dvm.encode_rotary(**good)) == 0
    for change in (dict(v=None), dict(v_cache=None), dict(k_out=k), dict(wq=torch.zeros(64)), dict(wq=torch.zeros(64), wk=torch.zeros(32)),
                   dict(angles=ang.double()), dict(angles=torch.zeros(64, 9).t()), dict(k=k.float()), dict(k_cache=cache.float()),
                   dict(k=k[:3]), dict(q_out=q[:, :, ::2])):
        with pytest.raises(dvm.DvmError):
            dvm.encode_rotary(**{**good, **change})


def launched(fn, d, places):
    """dvm_launch's status for tensors at these addresses: a refusal, or on a machine without a device its CUDA error."""
    st, buf, size = _encode(getattr(binding.lib, "dvm_encode_" + fn), d)
    assert st == OK
    return binding.lib.dvm_launch(buf, size, (C.c_void_p * len(places))(*places), len(places), None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are made up: only for a machine that cannot launch")
def test_outputs_that_overlap_are_refused():
    CUDA = -6
    far = [0x100000 * (i + 1) for i in range(16)]
    at = lambda n, **kw: [kw.get(f"t{i}", far[i]) for i in range(n)]   # noqa: E731
    # paging: cached, fresh, free, table, starts, lengths, positions, slots, taken; 5 requests, 100 rows, a table of 5 x 7
    assert launched("paging", paging(), at(9)) == CUDA
    assert launched("paging", paging(), at(9, t5=far[0])) == INVALID             # lengths over cached
    assert launched("paging", paging(), at(9, t5=far[0] + 16)) == INVALID        # its last element
    assert launched("paging", paging(), at(9, t5=far[0] + 20)) == CUDA           # just behind it
    assert launched("paging", paging(), at(9, t6=far[7] + 396)) == INVALID
    assert launched("paging", paging(free_pages=0), at(9, t8=far[2])) == CUDA    # an empty tensor overlaps nothing
    assert launched("paging", paging(), at(9, t1=far[0])) == CUDA                # inputs may
    # rotary, not paged, no norm: q, k, angles, positions, q_out, k_out
    kw = dict(norm=0, paged=0, k_out_stride=(128, 64))
    assert launched("rotary", rotary(**kw), at(6)) == CUDA
    assert launched("rotary", rotary(**kw), at(6, t4=far[0], t5=far[1])) == CUDA           # in place
    assert launched("rotary", rotary(**kw), at(6, t5=far[0])) == INVALID                   # keys over queries
    assert launched("rotary", rotary(**kw), at(6, t5=far[4])) == INVALID
    assert launched("rotary", rotary(**kw, q_out_stride=(512, 64)), at(6, t4=far[0])) == INVALID
    assert launched("rotary", rotary(**kw, out_dtype=0), at(6, t4=far[0])) == INVALID      # fp32 over bf16
    # attention: q, k, v, table, starts, lengths, out, workspace
    assert launched("attention", attention(), at(8)) == CUDA
    assert launched("attention", attention(), at(8, t2=far[1])) == CUDA                    # values in the keys' cache: inputs
    assert launched("attention", attention(), at(8, t6=far[0])) == INVALID
    assert launched("attention", attention(max_q=1), at(8, t7=far[6])) == INVALID          # the workspace over the output
