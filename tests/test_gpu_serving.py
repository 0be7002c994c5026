"""The serving operators on the GPU against their 64-bit definitions: sizes from nothing to long, odd sizes and strides,
masks that leave rows empty, what lies in hidden tokens, streams and graphs, and a run of them together."""
import math
import random

import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests import serving_oracle as orc
from tests.serving_oracle import f64

pytestmark = pytest.mark.gpu

F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


def ints(v):
    return torch.tensor(np.asarray(v), dtype=I32, device="cuda")


def normal(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=F32, device="cuda").normal_(0, std, generator=g).to(dtype)


def ok():
    torch.cuda.synchronize()
    assert dvm.last_device_status() == 0


# ------------------------------------------------------------------------------------------------------ paging

def run_paging(cached, fresh, free, table, page, rows):
    out = {"table": ints(table), "starts": ints(np.full(len(cached) + 1, 77)), "lengths": ints(np.full(len(cached), 77)),
           "positions": ints(np.full(rows, 77)), "slots": ints(np.full(rows, 77)), "taken": ints([77])}
    code = dvm.encode_paging(len(cached), table.shape[1], page, rows, len(free))
    dvm.launch(code, [ints(cached), ints(fresh), ints(free), out["table"], out["starts"], out["lengths"], out["positions"], out["slots"], out["taken"]])
    ok()
    want = orc.paging(cached, fresh, free, table, page, rows)
    for k, v in want.items():
        assert np.array_equal(out[k].cpu().numpy(), v), k


def paging_case(n, cached, fresh, page, seed, spare_blocks=2, pad=0, free_cut=0):
    r = np.random.default_rng(seed)
    c, f = r.integers(0, cached + 1, n), r.integers(0, fresh + 1, n)
    width = int(max(1, -(-(cached + fresh) // page) + spare_blocks))
    need = int((-(-(c + f) // page) - -(-c // page)).sum())
    pool = r.permutation(n * width + need + 5)
    table = pool[: n * width].reshape(n, width).copy()
    return c, f, pool[n * width: n * width + max(0, need - free_cut)], table, page, int(f.sum()) + pad


@pytest.mark.parametrize("n,cached,fresh,page,pad", [
    (1, 0, 1, 16, 0), (1, 100, 1, 16, 3), (32, 500, 1, 16, 0), (33, 70, 40, 8, 11), (257, 30, 5, 1, 0), (7, 3, 900, 128, 1),
    (256, 2048, 1024, 16, 173), (1000, 40, 3, 7, 5), (8192, 20, 4, 16, 9), (2, 0, 5000, 64, 0)])
def test_paging(n, cached, fresh, page, pad):
    run_paging(*paging_case(n, cached, fresh, page, n + fresh, pad=pad))


def test_paging_edges():
    none = np.zeros(0, np.int64)
    run_paging(none, none, none, np.zeros((0, 4), np.int64), 16, 5)                      # an empty batch: padding rows only
    run_paging(np.array([5]), np.array([0]), none, np.zeros((1, 2), np.int64), 16, 0)    # nothing new, no rows
    c, f, free, table, page, rows = paging_case(40, 60, 50, 16, 3, free_cut=6)
    run_paging(c, f, free, table, page, rows)                                            # the free pages run out
    run_paging(c, f, free[:0], table, page, rows)
    run_paging(c, f, free, table, page, rows - 77)                                       # more new tokens than rows
    run_paging(c, f, free, table[:, :3], page, rows)                                     # tables too narrow
    run_paging(c, f, free, np.zeros((40, 0), np.int64), page, rows)
    run_paging(c - 30, f - 20, free, np.where(table % 5, table, -1), page, rows)         # negative counts, holes in the table
    run_paging(np.array([2 ** 31 - 3, 4]), np.array([9, 2 ** 31 - 1]), free, table[:2], page, 12)


# ------------------------------------------------------------------------------------------------------ rotary

def angles(rows, rot, seed=1):
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))
    a = torch.arange(rows, dtype=torch.float64)[:, None] * inv[None]
    return torch.cat([a.cos(), a.sin()], 1).to(F32).cuda()


def check_rotary(t, hq, hk, dim, rot, dtype=BF16, out_dtype=None, w_dtype=None, norm=True, interleaved=False, paged=True, page=16, shift=0,
                 heads_first=False, seed=0, stream=None, huge=1.0):
    """shift: elements by which every tensor starts past a 16-byte boundary."""
    out_dtype, w_dtype = out_dtype or dtype, w_dtype or dtype
    rng = random.Random(seed)

    def moved(x):
        flat = torch.zeros(x.numel() + shift, dtype=x.dtype, device="cuda")
        flat[shift:] = x.reshape(-1)
        return flat[shift:].view(x.shape)

    qkv = moved(normal((t, hq + 2 * hk, dim), dtype, seed, huge))
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    wq, wk = (moved(1 + normal((dim,), w_dtype, seed + s, 0.1).float()).to(w_dtype) for s in (1, 2))
    ang = moved(angles(40 + t, rot))
    pos = [rng.randrange(40 + t) for _ in range(t)]
    pages = -(-t // page) + 1
    slots = list(range(pages * page))
    rng.shuffle(slots)
    slots = slots[:t]
    for i in range(t):
        if i % 5 == 3:
            pos[i] = rng.choice((-1, 40 + t, -(2 ** 31), 2 ** 31 - 1))   # a row that stays as it was
        if i % 7 == 4:
            slots[i] = rng.choice((-1, pages * page, 2 ** 31 - 1))       # a row that is not stored
    fill = 3.0
    q_out = moved(torch.full((t, hq, dim), fill, dtype=out_dtype, device="cuda"))
    shape = (pages, hk, page, dim) if heads_first else (pages, page, hk, dim)
    kc, vc = (moved(torch.full(shape, fill, dtype=out_dtype, device="cuda")) for _ in range(2))
    if heads_first:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    k_out = moved(torch.full((t, hk, dim), fill, dtype=out_dtype, device="cuda"))
    kw = dict(q=q, k=k, angles=ang, q_out=q_out, interleaved=interleaved, eps=1e-5)
    if norm:
        kw.update(wq=wq, wk=wk)
    kw.update(dict(v=v, k_cache=kc, v_cache=vc) if paged else dict(k_out=k_out))
    code = dvm.encode_rotary(**kw)
    ps, sl = ints(pos), ints(slots)
    launch = [q, k] + ([v] if paged else []) + ([wq, wk] if norm else []) + [ang, ps] + ([sl] if paged else []) + [q_out] + ([kc, vc] if paged else [k_out])
    torch.cuda.synchronize()
    dvm.launch(code, launch, stream)
    ok()
    eps_f = np.float64(np.float32(1e-5))
    Q, K, V, A = f64(q), f64(k), f64(v), f64(ang)
    want_q, want_k = np.full((t, hq, dim), fill), np.full((t, hk, dim), fill)
    mag_q, mag_k = np.zeros((t, hq, dim)), np.zeros((t, hk, dim))
    want_kc, want_vc, mag_kc = (np.full((pages * page, hk, dim), x) for x in (fill, fill, 0.0))
    for i in range(t):
        if not 0 <= pos[i] < 40 + t:
            continue
        for h in range(hq):
            want_q[i, h], mag_q[i, h] = orc.turn_head(Q[i, h], f64(wq) if norm else None, A[pos[i]], rot, eps_f, interleaved)
        for h in range(hk):
            want_k[i, h], mag_k[i, h] = orc.turn_head(K[i, h], f64(wk) if norm else None, A[pos[i]], rot, eps_f, interleaved)
        if 0 <= slots[i] < pages * page:
            want_kc[slots[i]], mag_kc[slots[i]], want_vc[slots[i]] = want_k[i], mag_k[i], V[i]
    # fp32 on the way: the sum of squares (dim roundings, halved by the root), root, quotient, weight, two products and a sum
    r = orc.EPS[out_dtype]
    step = (dim / 2 + 12) * 2.0 ** -24

    def near(got, want, mag):
        bad = np.abs(got - want) > r * np.abs(want) + step * mag * (1 + r)
        assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - want).max())

    near(f64(q_out), want_q, mag_q)
    if paged:
        near(f64(kc).reshape(-1, hk, dim), want_kc, mag_kc)
        near(f64(vc).reshape(-1, hk, dim), want_vc, 0 * want_vc)
    else:
        near(f64(k_out), want_k, mag_k)


@pytest.mark.parametrize("t,hq,hk,dim,rot", [(1, 1, 1, 8, 8), (1, 32, 32, 128, 128), (3, 5, 1, 64, 64), (37, 8, 2, 96, 48), (20, 4, 4, 80, 40),
                                             (9, 3, 1, 72, 24), (6, 2, 2, 256, 256), (5, 2, 1, 200, 64), (11, 40, 8, 128, 0), (400, 2, 1, 16, 8)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary(t, hq, hk, dim, rot, interleaved):
    check_rotary(t, hq, hk, dim, rot, interleaved=interleaved, seed=t)


@pytest.mark.parametrize("kw", [dict(dtype=F32), dict(dtype=F32, out_dtype=BF16), dict(out_dtype=F32, w_dtype=F32), dict(norm=False),
                                dict(paged=False), dict(paged=False, dtype=F32, norm=False), dict(shift=1), dict(shift=3, dtype=F32),
                                dict(heads_first=True), dict(page=1), dict(page=7), dict(page=128), dict(huge=1e4), dict(huge=1e-4)])
def test_rotary_variants(kw):
    check_rotary(23, 6, 2, 96, 64, seed=5, **kw)
    check_rotary(23, 6, 2, 80, 40, interleaved=True, seed=6, **kw)


def test_rotary_in_place_and_empty():
    q, k = normal((9, 4, 64), BF16, 1), normal((9, 2, 64), BF16, 2)
    ang, pos = angles(9, 64), ints(range(9))
    a, b = torch.empty_like(q), torch.empty_like(k)
    dvm.launch(dvm.encode_rotary(q=q, k=k, angles=ang, q_out=a, k_out=b), [q, k, ang, pos, a, b])
    dvm.launch(dvm.encode_rotary(q=q, k=k, angles=ang, q_out=q, k_out=k), [q, k, ang, pos, q, k])
    ok()
    assert torch.equal(a, q) and torch.equal(b, k)
    empty = q[:0]
    dvm.launch(dvm.encode_rotary(q=empty, k=k[:0], angles=ang, q_out=empty, k_out=k[:0]), [0, 0, ang, 0, 0, 0])
    dvm.launch(dvm.encode_rotary(q=q, k=k[:, :0], angles=ang, q_out=a, k_out=b[:, :0]), [q, 0, ang, pos, a, 0])   # no key heads
    ok()


# ------------------------------------------------------------------------------------------------------ attention

class Batch:
    def __init__(self, lengths, fresh, hq, hk, dim, page, dtype=BF16, heads_first=False, seed=0, spare=2, pad=0, std=1.0, shift=0):
        self.lengths, self.fresh = list(lengths), list(fresh)
        n, rows = len(self.lengths), int(sum(fresh)) + pad
        blocks = [-(-max(0, l) // page) for l in self.lengths]
        self.page, width, pages = page, max(blocks + [0]) + spare, sum(blocks) + 3
        r = np.random.default_rng(seed)
        ids = r.permutation(pages)
        table = np.full((n, width), -1)
        at = 0
        for i, b in enumerate(blocks):
            table[i, :b] = ids[at:at + b]
            at += b
        shape = (pages, hk, page, dim) if heads_first else (pages, page, hk, dim)
        self.k, self.v = normal(shape, dtype, seed + 1, std), normal(shape, dtype, seed + 2)
        if heads_first:
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        base = torch.zeros(rows * hq * dim + shift, dtype=dtype, device="cuda")
        self.q = base[shift:].view(rows, hq, dim)
        self.q.copy_(normal((rows, hq, dim), dtype, seed + 3, std))
        self.table, self.starts = ints(table), ints(np.concatenate([[0], np.cumsum(self.fresh)]))

    def code(self, out, **kw):
        return dvm.encode_attention(q=self.q, k_cache=self.k, v_cache=self.v, table=self.table, out=out, **kw)

    def launch(self, code, out, stream=None, workspace=None):
        if workspace is None:
            workspace = torch.full((max(16, dvm.tensor_extents(code)[-1]),), 0xff, dtype=torch.uint8, device="cuda")   # NaN
            torch.cuda.synchronize()
        dvm.launch(code, [self.q, self.k, self.v, self.table, self.starts, ints(self.lengths), out, workspace], stream)

    def check(self, window=0, sinks=0, max_q=None, scale=None, out_dtype=None, kernel=None, k=None, v=None):
        """Runs and compares; k, v: what the oracle reads in place of the cache."""
        dim = self.q.shape[-1]
        scale = scale or 1 / math.sqrt(dim)
        out = torch.full(self.q.shape, 7.0, dtype=out_dtype or self.q.dtype, device="cuda")
        code = self.code(out, scale=scale, window=window, sinks=sinks, max_q=max_q)
        self.launch(code, out)
        ok()
        if kernel and self.q.shape[0]:
            assert dvm.last_attention_kernel() == kernel
        want, mag, size, written, seen = orc.attention(f64(self.q), f64(self.k) if k is None else k, f64(self.v) if v is None else v,
                                                       self.table.cpu().numpy(), self.starts.cpu().numpy(), self.lengths,
                                                       float(np.float32(scale)), window, sinks, max_q or 1 << 30)
        got = f64(out)
        assert (got[~written] == 7.0).all()
        tol = orc.attention_bound(want, mag, size, seen, dim, out.dtype, self.q.dtype == BF16)
        bad = ~(np.abs(got - want) <= tol) & ~(np.isnan(got) & np.isnan(want))
        bad[~written] = False
        assert not bad.any(), (np.argwhere(bad)[:5], np.abs(got - want)[bad][:5], tol[bad][:5], bad.mean())
        return out


PROMPTS = [
    # lengths, fresh, hq, hk, dim, page, window, sinks
    ([1], [1], 1, 1, 64, 16, 0, 0),
    ([5], [5], 2, 1, 128, 16, 0, 0),
    ([130], [130], 4, 4, 128, 64, 0, 0),
    ([300, 1, 77], [300, 1, 77], 8, 2, 128, 16, 0, 0),
    ([700, 513, 64, 900], [100, 2, 64, 129], 8, 2, 64, 32, 0, 0),
    ([600, 300], [600, 300], 4, 2, 128, 16, 100, 4),
    ([600, 300, 0, 9], [70, 300, 0, 9], 5, 1, 96, 8, 33, 1),
    ([1000], [400], 14, 2, 80, 128, 257, 130),
    ([520], [520], 3, 3, 40, 256, 1, 0),
    ([400, 390], [9, 200], 33, 1, 128, 16, 64, 64),
    ([260, 10], [60, 10], 128, 1, 64, 16, 0, 0),
    ([50, 129], [50, 129], 6, 2, 8, 16, 20, 2),
]


@pytest.mark.parametrize("lengths,fresh,hq,hk,dim,page,window,sinks", PROMPTS)
@pytest.mark.parametrize("heads_first", [False, True])
def test_prompts(lengths, fresh, hq, hk, dim, page, window, sinks, heads_first):
    Batch(lengths, fresh, hq, hk, dim, page, heads_first=heads_first, seed=hq).check(window, sinks, max_q=max(max(fresh), 2))


SINGLES = [
    ([1], 1, 1, 64, 16, 0, 0), ([64], 8, 2, 128, 16, 0, 0), ([65], 8, 8, 128, 64, 0, 0), ([2049], 16, 1, 128, 16, 0, 0),
    ([5, 700, 64, 0, 129, 1000], 8, 2, 128, 16, 0, 0), ([900, 30, 513], 12, 4, 96, 8, 100, 4), ([900, 1, 513], 5, 1, 80, 128, 64, 70),
    ([3000, 2000], 4, 2, 64, 32, 1, 0), ([700] * 70, 3, 1, 40, 16, 333, 7), ([257, 258, 10], 34, 2, 128, 16, 0, 0), ([1500], 64, 8, 128, 256, 0, 0),
]


@pytest.mark.parametrize("lengths,hq,hk,dim,page,window,sinks", SINGLES)
@pytest.mark.parametrize("heads_first", [False, True])
def test_single_tokens(lengths, hq, hk, dim, page, window, sinks, heads_first):
    Batch(lengths, [1] * len(lengths), hq, hk, dim, page, heads_first=heads_first, seed=hq).check(window, sinks, max_q=1)


@pytest.mark.parametrize("kw", [dict(dtype=F32), dict(shift=1), dict(shift=4), dict(std=4.0), dict(std=0.01)])
@pytest.mark.parametrize("max_q", [1, 90])
def test_other_types_and_alignments(kw, max_q):
    b = Batch([90, 17, 300], [1, 1, 1] if max_q == 1 else [90, 17, 33], 6, 2, 64, 16, seed=3, **kw)
    b.check(window=50, sinks=3, max_q=max_q)
    b.check(max_q=max_q, out_dtype=F32)


def test_head_sizes_without_tensor_cores():
    Batch([90, 17], [90, 3], 2, 1, 33, 16).check(kernel="plain")
    Batch([90, 17], [1, 1], 2, 1, 256, 16).check(max_q=1, kernel="plain")


@pytest.mark.parametrize("single", [True, False])
def test_rows_that_see_nothing_and_rows_left_alone(single):
    # a length below the rows (positions before the first token), a length of nothing, holes in the table, rows behind the
    # last request, rows beyond max_q
    b = Batch([3, 0, 40, 100], [1, 1, 1, 1] if single else [9, 4, 40, 30], 4, 2, 64, 16, pad=5, seed=4)
    b.table[2, 1] = -1
    b.table[3, 0], b.table[3, 2] = 10 ** 9, -(2 ** 31)
    b.check(max_q=1 if single else 64)
    b.check(max_q=1 if single else 64, window=16)   # request 3: the window holds hidden pages only, for some rows
    b.check(max_q=1 if single else 20, window=3, sinks=20)
    b.lengths = [-5, 2 ** 31 - 1, 10 ** 6, 7]       # lengths that no table holds
    b.check(max_q=1 if single else 64)
    b.starts.copy_(ints([3, 2, 10 ** 8, -4, 5]))    # rows that overlap or do not exist: some request or none, nothing outside
    out = torch.zeros_like(b.q)
    b.launch(b.code(out, scale=1.0, max_q=1 if single else 64), out)
    ok()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), torch.finfo(BF16).min])
@pytest.mark.parametrize("single", [True, False])
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_what_hidden_tokens_hold_has_no_influence(single, bad, window, sinks):
    page, lengths = 16, [150, 37, 300]
    fresh = [1, 1, 1] if single else [150, 20, 130]
    b = Batch(lengths, fresh, 4, 2, 64, page, seed=8)
    clean_k, clean_v = f64(b.k), f64(b.v)
    hidden = []
    for i, l in enumerate(lengths):
        used = -(-l // page)
        hidden += [(int(b.table[i, used - 1]), s) for s in range(l - (used - 1) * page, page)]      # behind the last token
        if window:
            first = max(0, l - fresh[i] - window + 1)                                              # before every row's window
            hidden += [(int(b.table[i, s // page]), s % page) for s in range(sinks, first)]
    used_pages = set(int(p) for p in b.table.flatten() if p >= 0)
    hidden += [(p, s) for p in range(b.k.shape[0]) if p not in used_pages for s in range(page)]
    for p, s in hidden:
        b.k[p, s], b.v[p, s] = bad, bad
    out = b.check(window, sinks, max_q=1 if single else 150, k=clean_k, v=clean_v)
    assert torch.isfinite(out).all()
    if not single:
        # a bad value in a token that later rows see and earlier rows do not: only the later rows may know of it
        p, s = int(b.table[0, 4]), 6    # token 70 of request 0
        clean_out = out.clone()
        b.k[p, s, 1], b.v[p, s, 1] = bad, bad
        out2 = torch.full_like(out, 7.0)
        b.launch(b.code(out2, scale=1 / 8, window=window, sinks=sinks, max_q=150), out2)
        ok()
        want = orc.attention(f64(b.q), clean_k, clean_v, b.table.cpu().numpy(), b.starts.cpu().numpy(), lengths, 0.125, window, sinks)
        blind = [t for t in range(150) if t < 70 or (window and t >= 70 + window)]
        got, ref = f64(out2), want[0]
        tol = orc.attention_bound(want[0], want[1], want[2], want[4], 64, out.dtype, True)
        assert (np.abs(got[blind] - ref[blind]) <= tol[blind]).all()
        assert (np.abs(got[150:] - ref[150:]) <= tol[150:]).all()
        assert torch.equal(out2[:, :2], clean_out[:, :2])          # the other kv head
        if not math.isfinite(bad):
            assert not torch.isfinite(out2[70, 2:]).all()


@pytest.mark.parametrize("single", [True, False])
def test_strided_heads_and_outputs(single):
    b = Batch([100, 40], [1, 1] if single else [30, 40], 4, 2, 64, 16, seed=2)
    rows = b.q.shape[0]
    wide = torch.zeros((rows, 9, 64), dtype=BF16, device="cuda")     # query heads out of a wider row of heads
    wide[:, 3:7] = b.q
    b.q = wide[:, 3:7]
    b.check(max_q=1 if single else 40)
    out = torch.zeros((4, rows, 64), dtype=BF16, device="cuda").transpose(0, 1)
    dense = torch.zeros((rows, 4, 64), dtype=BF16, device="cuda")
    for o in (out, dense):
        b.launch(b.code(o, scale=0.125, max_q=1 if single else 40), o)
    odd = torch.zeros(rows * 4 * 65 + 1, dtype=BF16, device="cuda")[1:].view(rows, 4, 65)[:, :, :64]   # no 16-byte stores
    b.launch(b.code(odd, scale=0.125, max_q=1 if single else 40), odd)
    ok()
    assert torch.equal(out, dense) and torch.equal(odd, dense) and dense.abs().sum() > 0


@pytest.mark.parametrize("single", [True, False])
def test_streams_graphs_and_new_lengths(single):
    """A launch captured into a graph and replayed with other lengths and tables, on another stream than the eager runs."""
    fresh = [1, 1, 1] if single else [60, 33, 7]
    b = Batch([200, 90, 500], fresh, 8, 2, 128, 16, seed=6)
    out = torch.zeros_like(b.q)
    code = b.code(out, scale=0.1, max_q=1 if single else 60)
    ws = [torch.empty(max(16, dvm.tensor_extents(code)[-1]), dtype=torch.uint8, device="cuda") for _ in range(2)]
    lengths = ints([200, 90, 500])
    args = lambda o, w: [b.q, b.k, b.v, b.table, b.starts, lengths, o, w]   # noqa: E731
    dvm.launch(code, args(out, ws[0]))
    torch.cuda.synchronize()
    first = out.clone()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs, graphs = [torch.zeros_like(out), torch.zeros_like(out)], []
    for s, o, w in zip(side, outs, ws):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            dvm.launch(code, args(o, w), s)
        graphs.append(g)
    for _ in range(3):
        for s, g in zip(side, graphs):     # both at once, each with a workspace of its own
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], first) and torch.equal(outs[1], first)
    lengths.copy_(ints([150, 61, 499]))
    torch.cuda.synchronize()
    graphs[0].replay()
    dvm.launch(code, args(out, ws[1]), side[1])
    ok()
    assert torch.equal(outs[0], out) and not torch.equal(out, first)


def test_long_cache_offsets():
    """Pages beyond 2^32 elements of the cache (a view that skips most of it)."""
    page, hk, dim, pages = 16, 1, 64, 40
    step = 2 ** 27                                                       # elements between pages: 40 of them span 10 GB
    base = torch.empty(step * (pages - 1) + page * dim, dtype=BF16, device="cuda")
    view = base.as_strided((pages, page, hk, dim), (step, dim, dim, 1))
    view.copy_(normal((pages, page, hk, dim), BF16, 3))
    for fresh in ([1], [20]):
        b = Batch([600], fresh, 2, hk, dim, page, seed=4)
        b.k = b.v = view
        b.table.copy_(ints(np.random.default_rng(1).permutation(pages)[None]))
        b.check(max_q=fresh[0])


# ------------------------------------------------------------------------------------------------------ together

@pytest.mark.parametrize("window,sinks", [(0, 0), (48, 4)])
def test_a_step_after_the_other(window, sinks):
    """Prompts admitted, then tokens one by one: paging, rotary and attention as a serving loop runs them, against
    attention over each request's own keys in 64 bits."""
    n, hq, hk, dim, page, width = 3, 8, 2, 64, 16, 16
    pool = torch.randperm(60, device="cuda").to(I32)
    table = torch.full((n, width), -1, dtype=I32, device="cuda")
    kc, vc = (torch.full((60, page, hk, dim), float("nan"), dtype=BF16, device="cuda") for _ in range(2))
    wq, wk = (1 + normal((dim,), BF16, s, 0.1) for s in (1, 2))
    ang = angles(512, dim)
    cached, taken = np.zeros(n, np.int64), 0
    history = [[] for _ in range(n)]     # (k, v) of every token, 64 bits, after norm and rotation
    for step, fresh in enumerate([[33, 1, 0], [50, 0, 90], [1, 1, 1], [1, 1, 1], [1, 1, 1], [0, 1, 1]]):
        rows = int(sum(fresh)) + 4
        free = pool[taken:].contiguous()
        starts, lengths, pos, slots, took = (torch.full((m,), 77, dtype=I32, device="cuda") for m in (n + 1, n, rows, rows, 1))
        dvm.launch(dvm.encode_paging(n, width, page, rows, free.numel()),
                   [ints(cached), ints(fresh), free, table, starts, lengths, pos, slots, took])
        x = normal((rows, hq + 2 * hk, dim), BF16, 100 + step)
        q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        qr = torch.full((rows, hq, dim), 5.0, dtype=BF16, device="cuda")
        dvm.launch(dvm.encode_rotary(q=q, k=k, v=v, wq=wq, wk=wk, angles=ang, q_out=qr, k_cache=kc, v_cache=vc),
                   [q, k, v, wq, wk, ang, pos, slots, qr, kc, vc])
        out = torch.full_like(qr, 7.0)
        code = dvm.encode_attention(q=qr, k_cache=kc, v_cache=vc, table=table, out=out, scale=0.125, window=window, sinks=sinks, max_q=max(fresh))
        ws = torch.empty(max(16, dvm.tensor_extents(code)[-1]), dtype=torch.uint8, device="cuda")
        dvm.launch(code, [qr, kc, vc, table, starts, lengths, out, ws])
        ok()
        taken += int(took)
        K, V, Q, O, A = f64(k), f64(v), f64(qr), f64(out), f64(ang)
        t = 0
        for i in range(n):
            for j in range(fresh[i]):
                kk = np.stack([orc.turn_head(K[t + j, h], f64(wk), A[cached[i] + j], dim, np.float64(np.float32(1e-6)), False)[0] for h in range(hk)])
                history[i].append((kk, V[t + j]))
            for j in range(fresh[i]):
                p = int(cached[i]) + j
                s = [s for s in range(p + 1) if not window or s > p - window or s < sinks]
                for h in range(hq):
                    kh = np.stack([history[i][x][0][h // (hq // hk)] for x in s])
                    vh = np.stack([history[i][x][1][h // (hq // hk)] for x in s])
                    z = kh @ Q[t + j, h] * 0.125
                    w = np.exp(z - z.max())
                    w /= w.sum()
                    # the cached keys were rounded to bf16: scores off by 2^-8 of their magnitude, weights by twice that
                    ds = 2.0 ** -8 * (np.abs(kh) @ np.abs(Q[t + j, h])).max() * 0.125
                    tol = 2.0 ** -8 * np.abs(w @ vh) + (2.0 ** -8 + 2 * math.expm1(ds) + 1e-4) * (w @ np.abs(vh))
                    assert (np.abs(O[t + j, h] - w @ vh) <= tol).all(), (step, i, j, h)
            t += fresh[i]
        assert (O[t:] == 7.0).all() and (Q[t:] == 5.0).all()
        cached += np.array(fresh)
    assert (cached == [86, 5, 94]).all()
