"""The serving operators over the ranges their header allows, drawn by seed: sizes, layouts, masks, holes, lengths that do not fit."""
import random

import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests.test_gpu_serving import BF16, F32, Batch, check_rotary, ints, normal, ok, run_paging

pytestmark = pytest.mark.gpu

FAR = 2 ** 31 - 1


def layout(rng, x, dims):
    """The same values [.., D] behind other strides: dims in another order in memory, gaps behind rows of D, an offset of 16 bytes."""
    order = list(range(dims))
    rng.shuffle(order)
    gap, off = rng.choice((0, 0, 8, 24)), rng.choice((0, 8))
    shape = [x.shape[i] for i in order] + [x.shape[-1] + gap]
    flat = torch.full((int(np.prod(shape)) + off,), float("nan"), dtype=x.dtype, device="cuda")
    y = flat[off:].view(shape)[..., : x.shape[-1]].permute(*[order.index(i) for i in range(dims)], dims)
    y.copy_(x)
    return y


@pytest.mark.parametrize("seed", range(100))
def test_attention(seed):
    rng = random.Random(seed)
    single = rng.random() < 0.4
    hk = rng.choice((1, 1, 2, 3, 8))
    group = rng.choice((1, 2, 3, 4, 5, 7, 8, 11, 13, 16, 17, 21, 32, 64, 100, 127, 128) if hk == 1 else (1, 2, 3, 5, 8))
    dim = 8 * rng.randint(1, 16)
    page = rng.choice((8, 16, 32, 64, 128, 512))
    n = rng.choice((1, 1, 2, 3, 5, 33)) if group * hk <= 8 else rng.choice((1, 2, 3))
    most = 30 if n > 30 else 700 if group * hk <= 8 else 200
    lengths = [rng.randint(0, most) for _ in range(n)]
    fresh = [min(l, 1) if single else rng.randint(0, min(l, rng.choice((3, 90, 300)))) for l in lengths]
    b = Batch(lengths, fresh, group * hk, hk, dim, page, seed=seed, pad=rng.choice((0, 0, 3, 70)), std=rng.choice((0.1, 1.0, 2.0)))
    if b.q.shape[0] == 0:
        b = Batch(lengths + [5], fresh + [1], group * hk, hk, dim, page, seed=seed)
    b.q, b.k, b.v = layout(rng, b.q, 2), layout(rng, b.k, 3), layout(rng, b.v, 3)
    if rng.random() < 0.3:                              # holes
        for _ in range(3):
            b.table[rng.randrange(b.table.shape[0]), rng.randrange(b.table.shape[1])] = rng.choice((-1, b.k.shape[0], FAR, -FAR))
    if rng.random() < 0.2:                              # lengths that the rows or the table do not have
        b.lengths[rng.randrange(n)] = rng.choice((0, -7, 3, b.table.shape[1] * page, b.table.shape[1] * page + 40))
    window = rng.choice((0, 0, 1, 5, 64, 100, 333, FAR))
    sinks = rng.choice((0, 1, 4, 63, 64, 65, 200, FAR)) if window else rng.choice((0, 9))
    max_q = 1 if single else rng.choice((FAR, max(max(b.fresh), 2), max(max(b.fresh) // 2, 2)))
    kernel = "single" if single and group <= 16 else "prompt"
    b.check(window, sinks, max_q=max_q, scale=rng.choice((None, 0.3)), out_dtype=rng.choice((BF16, F32)), kernel=kernel)


@pytest.mark.parametrize("seed", range(40))
def test_rotary(seed):
    rng = random.Random(seed)
    dim = 8 * rng.randint(1, 32)
    hk = rng.choice((0, 1, 2, 5, 8))
    hq = rng.choice((0, 1, 3, 8, 40, 70)) if hk else rng.choice((1, 3, 40))
    check_rotary(rng.choice((1, 2, 17, 60)), hq, hk, dim, 8 * rng.randint(0, dim // 8), dtype=rng.choice((BF16, F32)), out_dtype=rng.choice((BF16, F32)),
                 w_dtype=rng.choice((BF16, F32)), norm=rng.random() < 0.7, interleaved=rng.random() < 0.5, paged=rng.random() < 0.6 and hk > 0,
                 page=rng.choice((1, 3, 16, 100)), shift=rng.choice((0, 0, 1, 4, 8)), heads_first=rng.random() < 0.5, seed=seed)


@pytest.mark.parametrize("seed", range(40))
def test_paging(seed):
    r = np.random.default_rng(seed)
    n, page, width = int(r.choice((0, 1, 5, 255, 256, 257, 700))), int(r.choice((1, 3, 16, 64, 1000, 400000))), int(r.choice((0, 1, 7, 40)))
    cached, fresh = r.integers(-3, 300, n), r.integers(-2, int(r.choice((2, 60))), n)
    rows = max(0, int(np.maximum(fresh, 0).sum()) + int(r.choice((0, 0, 9, -5, 1500))))
    free = r.permutation(5000)[: int(r.choice((0, 3, 4000)))]
    table = r.integers(-1, 5000, (n, width))
    run_paging(cached, fresh, free, table, page, rows)


def test_slots_that_pass_32_bits():
    """There is no page (-1) for a slot beyond 2^31 - 2, which no cache has."""
    page = 2 ** 30
    outs = [ints(np.full(m, 77)) for m in ((3, 1), 4, 3, 6, 6, 1)]
    outs[0].copy_(ints([[0], [1], [2]]))
    dvm.launch(dvm.encode_paging(3, 1, page, 6, 4), [ints([5, page - 2, 7]), ints([2, 2, 2]), ints(np.arange(4)), *outs])
    ok()
    assert outs[3].tolist() == [5, 6, page - 2, page - 1, 7, 8]
    assert outs[4].tolist() == [5, 6, 2 * page - 2, -1, -1, -1]


def test_sizes_of_nothing():
    q, kv = normal((3, 4, 64), BF16, 1), normal((2, 16, 2, 64), BF16, 2)
    for single in (True, False):
        max_q = 1 if single else 3
        out = torch.full_like(q, 7.0)
        # no blocks, no pages: every row sees nothing
        for cache, width in ((kv, 0), (kv[:0], 4), (kv[:0], 0)):
            table = torch.zeros((1, width), dtype=torch.int32, device="cuda")
            code = dvm.encode_attention(q=q, k_cache=cache, v_cache=cache, table=table, out=out, scale=1.0, max_q=max_q)
            ws = torch.empty(max(16, dvm.tensor_extents(code)[-1]), dtype=torch.uint8, device="cuda")
            out.fill_(7.0)
            dvm.launch(code, [q, cache.data_ptr() if cache.numel() else 0, cache.data_ptr() if cache.numel() else 0, table if width else 0,
                              ints([0, 3]), ints([900]), out, ws])
            ok()
            assert (out[:max_q] == 0).all() and (out[max_q:] == 7.0).all()
        # no requests, no rows
        table = torch.zeros((0, 4), dtype=torch.int32, device="cuda")
        code = dvm.encode_attention(q=q, k_cache=kv, v_cache=kv, table=table, out=out, scale=1.0, max_q=max_q)
        out.fill_(7.0)
        dvm.launch(code, [q, kv, kv, 0, ints([0]), 0, out, 0])
        code = dvm.encode_attention(q=q[:0], k_cache=kv, v_cache=kv, table=ints(np.zeros((1, 4))), out=out[:0], scale=1.0, max_q=max_q)
        dvm.launch(code, [0, kv, kv, ints(np.zeros((1, 4))), ints([0, 0]), ints([3]), 0, 0])
        ok()
        assert (out == 7.0).all()


def test_prompts_and_single_tokens_at_once():
    """The two kernels on two streams, in each other's way for shared and tensor memory, and in one graph after the other."""
    one = Batch([3000, 900, 64], [1, 1, 1], 8, 2, 64, 16, seed=1)
    many = Batch([700, 300], [700, 200], 8, 2, 64, 16, seed=2)
    sets = []
    for b, max_q in ((one, 1), (many, 700)):
        out = torch.zeros_like(b.q)
        code = b.code(out, scale=0.1, max_q=max_q)
        ws = torch.empty(max(16, dvm.tensor_extents(code)[-1]), dtype=torch.uint8, device="cuda")
        args = [b.q, b.k, b.v, b.table, b.starts, ints(b.lengths), out, ws]
        dvm.launch(code, args)
        ok()
        sets.append((code, args, out, out.clone(), torch.cuda.Stream()))
    for _ in range(30):
        for code, args, _, _, s in sets:
            dvm.launch(code, args, s.cuda_stream)
    ok()
    s = sets[0][4]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        for _ in range(3):
            for code, args, _, _, _ in sets:
                dvm.launch(code, args, s)
    for x in sets:
        x[2].zero_()
    torch.cuda.synchronize()
    g.replay()
    ok()
    for _, _, out, want, _ in sets:
        assert torch.equal(out, want) and want.abs().sum() > 0
