"""The operators of a layer of experts on the GPU against their 64-bit definitions: sizes from one to long, odd sizes and strides,
groups without rows, tokens that take no part, values that are not finite, streams and graphs, and a layer of them together."""
import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests import experts_oracle as orc
from tests.experts_oracle import f64

pytestmark = pytest.mark.gpu

F32, BF16, I32, U8, E4M3 = torch.float32, torch.bfloat16, torch.int32, torch.uint8, torch.float8_e4m3fn


def ints(v):
    return torch.tensor(np.asarray(v), dtype=I32, device="cuda")


def normal(shape, dtype, seed, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, dtype=F32, device="cuda").normal_(0, std, generator=g).to(dtype)


def ok():
    torch.cuda.synchronize()
    assert dvm.last_device_status() == 0


def spaced(shape, dtype, fill, pad):
    """A matrix whose rows are `pad` elements apart beyond their length."""
    return torch.full((shape[0], shape[1] + pad), fill, dtype=dtype, device="cuda")[:, :shape[1]]


def workspace(code):
    return torch.full((max(16, dvm.tensor_extents(code)[-1]),), 0xA5, dtype=U8, device="cuda")   # holds anything


# ------------------------------------------------------------------------------------------------------ routing

def run_routing(logits, top_k, scoring="softmax", bias=None, groups=1, top_groups=1, renormalise=False, factor=1.0, positions=None, stream=None):
    t, e = logits.shape
    out = [torch.full((t, top_k), 77, dtype=dt, device="cuda") for dt in (I32, F32, I32)] + [ints(np.full(e + 1, 77))]
    code = dvm.encode_routing(logits, top_k, scoring, bias is not None, groups, top_groups, renormalise, factor, positions is not None)
    dvm.launch(code, [logits] + ([bias] if bias is not None else []) + ([positions] if positions is not None else []) + out + [workspace(code)], stream)
    return out


def check_routing(logits, top_k, scoring="softmax", bias=None, groups=1, top_groups=1, renormalise=False, factor=1.0, positions=None):
    ids, weights, places, starts = (x.cpu().numpy() for x in run_routing(logits, top_k, scoring, bias, groups, top_groups, renormalise, factor, positions))
    ok()
    want = orc.routing(f64(logits), top_k, scoring, None if bias is None else f64(bias), groups, top_groups, renormalise, factor,
                       None if positions is None else positions.cpu().numpy())
    assert np.array_equal(ids, want[0])
    assert np.array_equal(places, want[2])
    assert np.array_equal(starts, want[3])
    w = want[1]
    assert np.array_equal(np.isnan(weights), np.isnan(w))
    fine = ~np.isnan(w)
    assert (np.abs(weights[fine] - w[fine]) <= np.abs(w[fine]) * orc.weights_bound(logits.shape[1]) + 2.0 ** -126).all()


@pytest.mark.parametrize("tokens", [1, 2, 31, 33, 64, 65, 700, 5000])
@pytest.mark.parametrize("experts,groups,top_groups,top_k,scoring,biased,dtype", [
    (64, 1, 1, 6, "softmax", False, BF16), (256, 8, 4, 8, "sigmoid", True, F32), (160, 8, 3, 6, "softmax", False, BF16), (8, 1, 1, 2, "softmax", True, F32)])
def test_routing(tokens, experts, groups, top_groups, top_k, scoring, biased, dtype):
    logits = normal((tokens, experts), dtype, tokens + experts, 1.5)
    bias = normal((experts,), F32, 3, 0.1) if biased else None
    positions = ints(np.where(np.arange(tokens) % 7 == 5, -1, np.arange(tokens)))
    check_routing(logits, top_k, scoring, bias, groups, top_groups, biased, 2.5 if biased else 1.0, positions)


@pytest.mark.parametrize("experts,groups,top_groups,top_k", [
    (1, 1, 1, 1), (2, 1, 1, 2), (3, 3, 2, 2), (33, 1, 1, 32), (32, 32, 32, 32), (512, 32, 1, 16), (512, 1, 1, 32), (511, 7, 2, 31), (100, 10, 10, 9), (257, 1, 1, 4), (64, 2, 2, 32)])
def test_routing_sizes(experts, groups, top_groups, top_k):
    for seed, (scoring, biased) in enumerate((("softmax", False), ("sigmoid", True), ("softmax", True), ("sigmoid", False))):
        logits = normal((70, experts + 3), BF16 if seed % 2 else F32, seed, 2.0)[:, :experts]     # rows apart, at odd addresses
        check_routing(logits, top_k, scoring, normal((experts,), F32, 9, 0.3) if biased else None, groups, top_groups, seed % 2 == 0, 0.5)


def test_routing_ties_and_near_ties():
    e, k = 128, 8
    same = torch.zeros((40, e), device="cuda")                                 # all equal: the first experts, of the first groups
    for scoring in ("softmax", "sigmoid"):
        for bias in (None, torch.zeros(e, device="cuda"), torch.full((e,), -0.25, device="cuda")):
            check_routing(same, k, scoring, bias)
            check_routing(same, k, scoring, bias, 8, 3)
    few = (normal((300, e), F32, 1) * 2).round().div(2)                        # few different values: many ties
    check_routing(few, k, "softmax")
    check_routing(few, k, "sigmoid", torch.zeros(e, device="cuda"), 4, 2)
    zeros = torch.where(torch.arange(e, device="cuda") % 2 == 0, 0.0, -0.0).expand(5, e).contiguous()
    check_routing(zeros, k)                                                    # 0 and -0 are equal
    # scores that 32 bits cannot tell apart: logits one step of fp32 from one another, and biases that undo what the logits do
    near = torch.full((200, e), 0.7, device="cuda").view(I32) + torch.randint(0, 6, (200, e), generator=torch.Generator("cuda").manual_seed(4), device="cuda", dtype=I32)
    near = near.view(F32)
    check_routing(near, k, "sigmoid", torch.zeros(e, device="cuda"))
    check_routing(near, k, "softmax", torch.zeros(e, device="cuda"), 8, 4)
    check_routing(near, k, "sigmoid", None, 8, 4)
    logits = normal((500, e), F32, 8, 1.0)
    bias = 0.5 - torch.sigmoid(logits[0])                                      # token 0: all values of c within a rounding of one another
    check_routing(logits, k, "sigmoid", bias)
    check_routing(logits, 32, "sigmoid", bias, 4, 3)


def test_routing_values_that_are_not_finite():
    e, inf, nan = 64, float("inf"), float("nan")
    base = normal((40, e), F32, 5)
    for value in (-inf, torch.finfo(F32).min, torch.finfo(F32).max):
        x = base.clone()
        x[::2, 3:50] = value
        for scoring in ("softmax", "sigmoid"):
            check_routing(x, 6, scoring)
            check_routing(x, 6, scoring, groups=8, top_groups=5)
            check_routing(x, 6, scoring, torch.zeros(e, device="cuda"))
    for bad in (nan, inf):
        x = base.clone()
        x[1, 5], x[3, :], x[7, 60:] = bad, bad, bad
        check_routing(x, 6, "softmax")
        check_routing(x, 6, "sigmoid", torch.zeros(e, device="cuda"))
    bias = normal((e,), F32, 6, 0.1)
    bias[10:30] = -inf                                                         # experts that are switched off
    bias[40] = inf
    check_routing(base, 6, "sigmoid", bias)
    bias[2] = nan                                                              # counts less than any other
    check_routing(base, 64 // 2, "sigmoid", bias)
    x = base.clone()
    x[0, 2], x[5, :8] = nan, nan
    check_routing(x, 4, "sigmoid", None, 8, 3)


def test_routing_of_no_token_and_of_none_that_takes_part():
    code = dvm.encode_routing(torch.empty((0, 16), device="cuda"), 4)
    starts = ints(np.full(17, 77))
    empty = torch.empty(0, device="cuda")
    dvm.launch(code, [empty, empty, empty, empty, starts, empty])
    ok()
    assert (starts == 0).all()
    for tokens in (40, 200):
        check_routing(normal((tokens, 16), F32, 1), 4, positions=ints(np.full(tokens, -1)))
        check_routing(normal((tokens, 16), F32, 1), 4, positions=ints(np.where(np.arange(tokens) == tokens - 1, 0, -5)))


def test_routing_of_many_tokens():
    """Chunks of several rounds; every expert's rows in the tokens' order (checked without the loop of the 64-bit form)."""
    t, e, k = 40000, 64, 4
    logits = normal((t, e), F32, 3)
    ids, weights, places, starts = run_routing(logits, k)
    ok()
    want = logits.double().sort(dim=1, descending=True, stable=True)[1][:, :k]
    assert torch.equal(ids.long(), want)
    by_expert, order = ids.reshape(-1).long().sort(stable=True)
    rows = torch.empty_like(order)
    rows[order] = torch.arange(t * k, device="cuda")
    assert torch.equal(places.reshape(-1).long(), rows)
    assert torch.equal(starts.long(), torch.searchsorted(by_expert, torch.arange(e + 1, device="cuda")))


@pytest.mark.parametrize("t,e,k,alike", [(592 * 16, 33, 3, False), (592 * 16 + 1, 200, 2, True), (592 * 240, 8, 1, True), (592 * 240 + 1, 16, 2, True),
                                         (1200001, 5, 2, True), (200000, 512, 1, False), (700003, 40, 2, True)])
def test_routing_of_more_chunks(t, e, k, alike):
    """More tokens than the chunks of one launch's size; with `alike` all of a chunk's tokens are at the same expert, the most that it counts."""
    g = torch.Generator("cuda").manual_seed(t)
    logits = torch.randn((1 if alike else t, e), generator=g, device="cuda").expand(t, e).contiguous()
    ids, weights, places, starts = run_routing(logits, k)
    ok()
    assert torch.equal(ids.long(), logits.sort(dim=1, descending=True, stable=True)[1][:, :k])
    by_expert, order = ids.reshape(-1).long().sort(stable=True)
    rows = torch.empty_like(order)
    rows[order] = torch.arange(t * k, device="cuda")
    assert torch.equal(places.reshape(-1).long(), rows)
    assert torch.equal(starts.long(), torch.searchsorted(by_expert, torch.arange(e + 1, device="cuda")))


# ------------------------------------------------------------------------------------------------------ quantize

def check_quantize(x, gated=False, copies=0, block_rows=1, pad=16, seed=0, some_outside=False):
    rows, cols = x.shape[0], x.shape[1] // (2 if gated else 1)
    out_rows = rows * copies + 3 if copies else rows
    codes = spaced((out_rows, cols), U8, 0x11, pad)
    scales = spaced((-(-out_rows // block_rows), -(-cols // 128)), F32, 7.0, 3)
    places = None
    if copies:
        places = np.random.default_rng(seed).permutation(out_rows)[: rows * copies].reshape(rows, copies)
        if some_outside:
            places[::3, 0] = -1
            places[1::3, copies - 1] = out_rows
            places[2::3, copies // 2] = 2 ** 31 - 1
    code = dvm.encode_quantize(x, codes, scales, None if places is None else ints(places), gated, block_rows)
    dvm.launch(code, [x] + ([] if places is None else [ints(places)]) + [codes, scales])
    ok()
    got_codes, got_scales = codes.cpu().numpy(), f64(scales)
    v = f64(x)
    if gated:
        with np.errstate(over="ignore", invalid="ignore"):
            v = v[:, :cols] / (1.0 + np.exp(-v[:, :cols])) * v[:, cols:]
    want_codes, want_scales = np.full((out_rows, cols), 0x11), np.full(got_scales.shape, 7.0)
    c, s = orc.quantize(v, block_rows)
    index = np.arange(rows)[:, None] if places is None else places
    for j in range(index.shape[1]):
        in_range = (index[:, j] >= 0) & (index[:, j] < out_rows)
        want_codes[index[in_range, j]] = c[in_range]
        if block_rows == 1:
            want_scales[index[in_range, j]] = s[in_range]
    if block_rows > 1:
        want_scales = s
    if not gated:
        assert np.array_equal(got_scales, want_scales, equal_nan=True)
        assert np.array_equal(got_codes, want_codes)
        return
    # v in fp32: silu's exponential (2 ulp and its argument's rounding, |z| 2^-24), a sum, a quotient (2 ulp) and a product
    assert np.array_equal(np.isnan(got_scales), np.isnan(want_scales))
    fine = ~np.isnan(want_scales)
    z = np.abs(f64(x)[:, :cols]).max(initial=0.0) if np.isfinite(f64(x)).all() else 100.0
    rel = (4 + 2 * z + 2 + 4 + 2) * 2.0 ** -24
    assert (np.abs(got_scales - want_scales)[fine] <= rel * want_scales[fine] + 2.0 ** -149).all()
    # each code's value within half a step of v over the scale that was written; a step is 2^-3 of the value's power of two, 2^-9 at least
    for j in range(index.shape[1]):
        for r in range(rows):
            to = index[r, j]
            if not 0 <= to < out_rows:
                continue
            sc = np.repeat(got_scales[to], 128)[:cols]
            good = ~np.isnan(sc)
            q = v[r][good] / sc[good]
            step = 2.0 ** np.maximum(np.floor(np.log2(np.maximum(np.abs(q), 1e-30))) - 3, -9)
            err = np.abs(orc.decode(got_codes[to][good]) - q)
            assert (err <= step / 2 + 2 * rel * np.abs(q) + 2.0 ** -130 / sc[good]).all()
            assert (got_codes[to][~good] == 0).all()
    untouched = np.setdiff1d(np.arange(out_rows), index[(index >= 0) & (index < out_rows)])
    assert (got_codes[untouched] == 0x11).all() and (got_scales[untouched] == 7.0).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,copies,shift", [(1, 16, 0, 0), (1, 4096, 8, 0), (3, 144, 1, 0), (70, 1408, 6, 0), (257, 128, 0, 1), (64, 2000, 3, 3), (33, 272, 32, 2), (2000, 256, 2, 0)])
def test_quantize(dtype, rows, cols, copies, shift):
    x = normal((rows, cols + 8 + shift), dtype, rows + cols) * torch.exp(normal((cols + 8 + shift,), dtype, 1))
    check_quantize(x[:, shift: shift + cols], copies=copies, some_outside=copies > 1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,copies,shift", [(1, 16, 0, 0), (130, 1408, 0, 0), (7, 272, 2, 1), (65, 144, 0, 3)])
def test_quantize_gated(dtype, rows, cols, copies, shift):
    x = normal((rows, 2 * cols + 8 + shift), dtype, rows + cols, 3.0)
    check_quantize(x[:, shift: shift + 2 * cols], gated=True, copies=copies)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols,shift", [(1, 16, 0), (128, 128, 0), (129, 144, 0), (300, 1408, 0), (77, 272, 1)])
def test_quantize_weights(dtype, rows, cols, shift):
    x = normal((rows, cols + 8 + shift), dtype, rows + cols, 0.02)
    check_quantize(x[:, shift: shift + cols], block_rows=128)


def test_quantize_borders():
    """Quotients on the borders between two codes and a step of fp32 beside them, for scales that are not powers of two."""
    t = orc.e4m3_values()
    edges = np.concatenate([(t[1:] + t[:-1]) / 2, t[1:]])
    rows = []
    for top in (448.0, 1.0, 3.0, 447.0, 1e-3, 2.0 ** -110, 1e30):
        s = orc.scale_of(np.array([np.float32(top)]))[0]
        at = (edges * s).astype(np.float32)
        for delta in (-2, -1, 0, 1, 2):
            v = (at.view(np.int32) + delta).view(np.float32)
            v = v[np.abs(v) < top]
            for i in range(0, len(v), 126):
                row = np.zeros(128, np.float32)
                row[: len(v[i: i + 126])] = v[i: i + 126]
                row[126], row[127] = top, -top
                rows += [row, -row]
    x = torch.tensor(np.stack(rows), device="cuda")
    check_quantize(x)
    check_quantize(x[:64], block_rows=128)
    # bf16 quotients of small numbers: borders without end
    x = torch.randint(-200, 201, (300, 256), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(BF16)
    x[:, 0] = 56 * 4
    x[::2, 128] = 255
    check_quantize(x)
    check_quantize(x.float(), block_rows=128)


def test_quantize_small_large_and_not_finite():
    inf, nan = float("inf"), float("nan")
    x = normal((60, 384), F32, 2)
    x[0] = 0.0
    x[1] = -0.0
    x[2] *= 1e-38                       # subnormal values and a scale of 2^-126
    x[3] *= 1e-44
    x[4] = torch.finfo(F32).max
    x[5, 7], x[6, 140], x[7, 383] = inf, -inf, nan
    x[8, :128] = 2.0 ** -126 * 448
    x[9, :128] = 2.0 ** -130
    for dtype in (F32, BF16):
        y = x.to(dtype)
        check_quantize(y)
        check_quantize(y, copies=2)
        check_quantize(y[8:], block_rows=128)
        check_quantize(y, block_rows=128)
    g = torch.cat([x, normal((60, 384), F32, 3)], 1)
    g[4] = 1.0
    g[20, 3], g[21, 3], g[22, 3] = -200.0, 200.0, -88.0
    check_quantize(g, gated=True)


# ------------------------------------------------------------------------------------------------------ scaled matmul

def small_codes(shape, seed):
    """Codes of the values -2 .. 2 and powers of two as scales: every sum is exact, in whatever order."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(F32).to(E4M3)


def small_scales(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.exp2(torch.randint(-1, 2, shape, generator=g, device="cuda").to(F32))


def any_codes(shape, seed):
    return normal(shape, F32, seed, 60.0).clamp(-448, 448).to(E4M3)


def values(codes, scales, block_rows):
    """64-bit values of codes [..., rows, cols]."""
    wide = scales.double().repeat_interleave(128, -1)[..., : codes.shape[-1]]
    if block_rows > 1:
        wide = wide.repeat_interleave(128, -2)[..., : codes.shape[-2], :]
    return codes.to(F32).double() * wide


def check_scaled(counts, n, k, dtype=BF16, exact=True, pad=0, grouped=True, behind=3, seed=0, stream=None, starts=None, x_pad=0):
    """behind: rows behind the last group."""
    groups, rows = len(counts), int(np.sum(counts)) + (behind if grouped else 0)
    make, scale = (small_codes, small_scales) if exact else (any_codes, lambda s, i: normal(s, F32, i).abs() + 0.01)
    x = make((rows, k + x_pad), seed)[:, :k]
    w = make((groups, n + 1, k + x_pad), seed + 1)[:, :n, :k]
    xs, ws = scale((rows, -(-k // 128) + 2), seed + 2)[:, : -(-k // 128)], scale((groups, -(-n // 128), -(-k // 128)), seed + 3)
    out = spaced((rows, n), dtype, 7.0, pad)
    first = np.concatenate([[0], np.cumsum(counts)]) if starts is None else starts
    st = ints(first) if grouped else None
    code = dvm.encode_scaled_matmul(x, xs, w, ws, out, st)
    torch.cuda.synchronize()
    dvm.launch(code, [x, xs, w, ws] + ([st] if grouped else []) + [out, workspace(code)], stream)
    ok()
    X, W = values(x, xs, 1), values(w, ws, 128)
    want, mag = torch.full((rows, n), 7.0, dtype=torch.float64, device="cuda"), torch.zeros((rows, n), dtype=torch.float64, device="cuda")
    touched = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for g in range(groups):
        a, b = (min(max(int(v), 0), rows) for v in (first[g], first[g + 1])) if grouped else (0, rows)
        if b > a:
            want[a:b], mag[a:b] = X[a:b] @ W[g].T, X[a:b].abs() @ W[g].abs().T
            touched[a:b] = True
    got = out.double()
    if exact:
        assert float(mag.max()) < 2 ** 22
        assert torch.equal(got, torch.where(touched[:, None], want.to(dtype).double(), want))
    else:
        bound = orc.scaled_bound(want.cpu().numpy(), mag.cpu().numpy(), -(-k // 128), dtype)
        err = (got - want).abs().cpu().numpy()
        assert (err[touched.cpu().numpy()] <= bound[touched.cpu().numpy()]).all()
        assert bool((got[~touched] == 7.0).all())
    return out


def uneven(rows, groups, seed):
    r = np.random.default_rng(seed)
    p = np.exp(r.standard_normal(groups))
    c = r.multinomial(rows, p / p.sum())
    c[seed % groups] = 0
    return c


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 32, 33, 64, 65, 128, 129, 300, 700])
@pytest.mark.parametrize("n,k", [(128, 128), (200, 272), (1000, 1408), (8, 16), (257, 4096)])
def test_scaled_dense(rows, n, k):
    check_scaled([rows], n, k, BF16 if rows % 2 else F32, grouped=False)


@pytest.mark.parametrize("rows,groups", [(1, 1), (1, 9), (20, 8), (60, 33), (500, 64), (500, 20), (900, 8), (40, 200), (3000, 5)])
@pytest.mark.parametrize("n,k", [(200, 272), (640, 1024)])
def test_scaled_groups(rows, groups, n, k):
    check_scaled(uneven(rows, groups, rows + groups) if groups > 1 else [rows], n, k, F32 if rows % 3 else BF16, pad=rows % 2 * 3)


def test_scaled_shapes():
    check_scaled([5, 0, 0, 130, 1], 40, 48, pad=1, x_pad=16)                # strides beyond the rows, odd output rows
    check_scaled([0, 0, 0], 200, 272)                                       # no group has a row: nothing is written
    check_scaled([0] * 1000 + [3] + [0] * 23, 130, 160)                     # many groups, one in use
    check_scaled([1] * 1024, 72, 144)
    check_scaled([2, 3], 20000, 128, F32)                                   # wide: more tiles than CTAs
    check_scaled([3], 128, 16384, F32)                                      # long: one tile over all CTAs
    check_scaled([7], 130, 12000, grouped=False)
    check_scaled([2000, 1, 0, 1500], 384, 640)


@pytest.mark.parametrize("rows,groups,n,k,dtype", [(1, 1, 1000, 4096, F32), (50, 8, 300, 2000, F32), (400, 3, 700, 1408, BF16), (2000, 4, 512, 512, F32), (40, 1, 260, 272, BF16)])
def test_scaled_values(rows, groups, n, k, dtype):
    check_scaled(uneven(rows, groups, 1) if groups > 1 else [rows], n, k, dtype, exact=False, seed=rows)


def test_scaled_starts_that_make_no_sense_stay_inside():
    """Descending, negative and far starts: what they cut out is computed, the rest stays; no two groups overlap here."""
    check_scaled([10, 10, 10, 10], 136, 144, starts=np.array([-5, 7, 7, 30, 2 ** 31 - 1]))
    check_scaled([10, 10, 10, 10], 136, 144, starts=np.array([20, 10, 20, 35, -(2 ** 31)]))
    check_scaled([100, 300], 136, 144, starts=np.array([500, 600, 900]))


def test_scaled_rows_do_not_depend_on_others():
    """NaN codes and scales of other rows, groups and rows behind the last group leave a row's bits alone."""
    n, k, counts = 300, 1408, [40, 30, 50]
    first = np.concatenate([[0], np.cumsum(counts)])
    x, w = any_codes((125, k), 1), any_codes((3, n, k), 2)
    xs, ws = normal((125, 11), F32, 3).abs(), normal((3, 3, 11), F32, 4).abs()
    out = torch.zeros((125, n), device="cuda")
    code = dvm.encode_scaled_matmul(x, xs, w, ws, out, ints(first))
    work = workspace(code)
    dvm.launch(code, [x, xs, w, ws, ints(first), out, work])
    ok()
    want = out.clone()
    x.view(U8)[[3, 75, 121]] = 0x7f
    xs[5], xs[123] = float("nan"), float("inf")
    w.view(U8)[2] = 0xff
    out.fill_(7.0)
    dvm.launch(code, [x, xs, w, ws, ints(first), out, work])
    ok()
    for r in range(125):
        if r >= 120:
            assert bool((out[r] == 7.0).all()), r
        elif r in (3, 5) or r >= 70:
            assert bool(out[r].isnan().all()), r
        else:
            assert torch.equal(out[r], want[r]), r


# ------------------------------------------------------------------------------------------------------ combine

def check_combine(tokens, k, rows, cols, dtype=BF16, based=True, pad=0, shift=0, in_place=False, seed=0):
    y = normal((rows, cols + pad + shift), dtype, seed)[:, shift: shift + cols]
    r = np.random.default_rng(seed)
    places = r.integers(0, max(rows, 1), (tokens, k))
    places[::4, 0] = -1
    places[1::5] = r.choice([-1, rows, 2 ** 31 - 1, -(2 ** 31)], (len(places[1::5]), k))     # tokens without any row
    weights = normal((tokens, k), F32, seed + 1)
    base = normal((tokens, cols + pad + shift), dtype, seed + 2)[:, shift: shift + cols]
    before = f64(base) if in_place else np.full((tokens, cols), 7.0)
    want, mag, any_row = orc.combine(f64(y), places, f64(weights), f64(base) if based else None)
    out = base if in_place else torch.full((tokens, cols + pad + shift), 7.0, dtype=dtype, device="cuda")[:, shift: shift + cols]
    code = dvm.encode_combine(y, ints(places), weights, out, base if based else None)
    dvm.launch(code, [y, ints(places), weights] + ([base] if based else []) + [out])
    ok()
    got = f64(out)
    assert np.array_equal(got[~any_row], before[~any_row])
    assert (np.abs(got - want)[any_row] <= orc.combine_bound(want, mag, k, dtype)[any_row]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,k,cols", [(1, 1, 8), (1, 8, 4096), (64, 6, 4096), (37, 9, 1000), (300, 32, 72), (5, 3, 3), (1000, 8, 256)])
def test_combine(dtype, tokens, k, cols):
    check_combine(tokens, k, tokens * k + 5, cols, dtype, based=tokens % 2 == 1)
    check_combine(tokens, k, tokens, cols, dtype, based=tokens % 2 == 0, pad=5, shift=1)
    check_combine(tokens, k, tokens, cols, dtype, pad=8, in_place=True)


def test_combine_of_nothing():
    check_combine(3, 2, 0, 16)     # no rows at all: nothing is written
    code = dvm.encode_combine(torch.zeros((4, 16), device="cuda"), ints(np.zeros((0, 2))), torch.zeros((0, 2), device="cuda"), torch.zeros((0, 16), device="cuda"))
    dvm.launch(code, [torch.zeros((4, 16), device="cuda")] * 4)
    ok()


# ------------------------------------------------------------------------------------------------------ together

class Layer:
    """A layer of experts as it is used: codes encoded once for the batch's size, tensors the caller's own."""

    def __init__(self, tokens, hidden, inner, experts, top_k, seed=0):
        self.t, self.h, self.f, self.e, self.k = tokens, hidden, inner, experts, top_k
        rows = tokens * top_k
        kb = lambda n: -(-n // 128)   # noqa: E731
        z = lambda *s, dtype=F32: torch.zeros(s, dtype=dtype, device="cuda")   # noqa: E731
        up, down = normal((experts, 2 * inner, hidden), BF16, seed, hidden ** -0.5), normal((experts, hidden, inner), BF16, seed + 1, inner ** -0.5)
        self.wu, self.wus = z(experts, 2 * inner, hidden, dtype=E4M3), z(experts, kb(2 * inner), kb(hidden))
        self.wd, self.wds = z(experts, hidden, inner, dtype=E4M3), z(experts, kb(hidden), kb(inner))
        for g in range(experts):
            for w, c, s in ((up, self.wu, self.wus), (down, self.wd, self.wds)):
                dvm.launch(dvm.encode_quantize(w[g], c[g], s[g], block_rows=128), [w[g], c[g], s[g]])
        self.bias = normal((experts,), F32, seed + 2, 0.05)
        self.logits, self.x, self.positions, self.out = z(tokens, experts), z(tokens, hidden, dtype=BF16), z(tokens, dtype=I32), z(tokens, hidden, dtype=BF16)
        self.ids, self.places, self.weights, self.starts = z(tokens, top_k, dtype=I32), z(tokens, top_k, dtype=I32), z(tokens, top_k), z(experts + 1, dtype=I32)
        self.xc, self.xs, self.y = z(rows, hidden, dtype=E4M3), z(rows, kb(hidden)), z(rows, 2 * inner, dtype=BF16)
        self.gc, self.gs, self.yd = z(rows, inner, dtype=E4M3), z(rows, kb(inner)), z(rows, hidden, dtype=BF16)
        self.route = dvm.encode_routing(self.logits, top_k, "sigmoid", True, 2, 1, True, 2.5, True)
        self.spread = dvm.encode_quantize(self.x, self.xc, self.xs, self.places)
        self.up = dvm.encode_scaled_matmul(self.xc, self.xs, self.wu, self.wus, self.y, self.starts)
        self.gate = dvm.encode_quantize(self.y, self.gc, self.gs, gated=True)
        self.down = dvm.encode_scaled_matmul(self.gc, self.gs, self.wd, self.wds, self.yd, self.starts)
        self.join = dvm.encode_combine(self.yd, self.places, self.weights, self.out, self.x)
        self.work = [workspace(c) for c in (self.route, self.up, self.down)]

    def run(self, stream=None):
        dvm.launch(self.route, [self.logits, self.bias, self.positions, self.ids, self.weights, self.places, self.starts, self.work[0]], stream)
        dvm.launch(self.spread, [self.x, self.places, self.xc, self.xs], stream)
        dvm.launch(self.up, [self.xc, self.xs, self.wu, self.wus, self.starts, self.y, self.work[1]], stream)
        dvm.launch(self.gate, [self.y, self.gc, self.gs], stream)
        dvm.launch(self.down, [self.gc, self.gs, self.wd, self.wds, self.starts, self.yd, self.work[2]], stream)
        dvm.launch(self.join, [self.yd, self.places, self.weights, self.x, self.out], stream)

    def fill(self, real, seed):
        self.logits.copy_(normal((self.t, self.e), F32, seed, 1.5))
        self.x.copy_(normal((self.t, self.h), BF16, seed + 1))
        self.positions.copy_(torch.where(torch.arange(self.t, device="cuda") < real, 0, -1))
        self.out.fill_(7.0)

    def check(self, real):
        """Against the definitions, from the weights' and activations' own codes; the steps' roundings are followed: the bf16 product's
        (2^-8 of |y|), the gate's codes (2^-4 of each value, or 2^-10 of its block's scale), the second product's and the sum's."""
        ids, weights, places, starts = orc.routing(f64(self.logits), self.k, "sigmoid", f64(self.bias), 2, 1, True, 2.5, self.positions.cpu().numpy())
        assert np.array_equal(self.ids.cpu().numpy(), ids) and np.array_equal(self.places.cpu().numpy(), places) and np.array_equal(self.starts.cpu().numpy(), starts)
        x, out = f64(self.x), f64(self.out)
        xc, xs = orc.quantize(x)
        X = orc.decode(xc) * np.repeat(xs, 128, 1)[:, : self.h]
        WU, WD = values(self.wu, self.wus, 128).cpu().numpy(), values(self.wd, self.wds, 128).cpu().numpy()
        for t in range(self.t):
            if t >= real:
                assert (out[t] == 7.0).all()
                continue
            want, err = x[t].copy(), np.zeros(self.h)
            for j in range(self.k):
                e = ids[t, j]
                y = WU[e] @ X[t]
                # (the gate and up values' own error, e_y, through silu(g) u: |silu'| is at most 1.1)
                ey = orc.scaled_bound(y, np.abs(WU[e]) @ np.abs(X[t]), 1 + self.h // 128, BF16)
                g, u = y[: self.f], y[self.f:]
                s = g / (1 + np.exp(-g))
                v, ev = s * u, 1.1 * ey[: self.f] * np.abs(u) + (np.abs(s) + 1.1 * ey[: self.f]) * ey[self.f:]
                top = np.repeat([np.abs(v[b: b + 128]).max() + ev[b: b + 128].max() for b in range(0, self.f, 128)], 128)[: self.f]
                ev = ev + np.maximum((np.abs(v) + ev) * 2.0 ** -4, top / 448 * 2.0 ** -10) * (1 + 2.0 ** -20)
                z = WD[e] @ v
                ez = np.abs(WD[e]) @ ev
                ez = ez + orc.scaled_bound(z, np.abs(WD[e]) @ (np.abs(v) + ev), 1 + self.f // 128, BF16) + 2.0 ** -8 * ez
                want += weights[t, j] * z
                err += weights[t, j] * (ez + np.abs(z) * 2.0 ** -18)
            assert (np.abs(out[t] - want) <= err + 2.0 ** -8 * (np.abs(want) + err) + 1e-6).all(), t


@pytest.mark.parametrize("tokens,real,hidden,inner,experts,top_k", [(1, 1, 256, 144, 8, 2), (5, 4, 272, 128, 16, 4), (90, 83, 512, 192, 8, 2), (400, 400, 256, 256, 4, 2)])
def test_a_layer(tokens, real, hidden, inner, experts, top_k):
    layer = Layer(tokens, hidden, inner, experts, top_k)
    for step in range(2):
        layer.fill(real, 10 * step)
        layer.run()
        ok()
        layer.check(real)


def test_a_layer_captured_and_replayed_with_other_plans():
    layer = Layer(60, 256, 192, 16, 4)
    layer.fill(60, 1)
    layer.run()
    ok()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.run(side)
    for step, real in enumerate((60, 1, 37)):
        layer.fill(real, 20 + step)
        graph.replay()
        ok()
        layer.check(real)


def test_layers_on_two_streams_at_once():
    a, b = Layer(70, 256, 192, 8, 2), Layer(200, 512, 128, 8, 4, seed=5)
    a.fill(66, 1)
    b.fill(200, 2)
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        a.run(one)
        b.run(two)
    ok()
    a.check(66)
    b.check(200)


def test_launches_wait_for_what_comes_before():
    """Inputs that the kernels just before on the stream write: library launches and others in turn."""
    layer = Layer(64, 256, 128, 8, 2)
    layer.fill(64, 3)
    layer.run()
    ok()
    want = layer.out.clone()
    x, logits = layer.x.clone(), layer.logits.clone()
    for _ in range(10):
        layer.x.zero_()
        layer.logits.zero_()
        layer.run()
        layer.x.copy_(x)
        layer.logits.copy_(logits)
        layer.run()
    ok()
    assert torch.equal(layer.out, want)
