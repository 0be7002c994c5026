"""Drawn calls of the operators of a layer of experts against their 64-bit definitions: sizes, strides, types, offsets of the first
value, plans with uneven groups; and which of the scaled product's kernels takes which sizes."""
import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests import experts_oracle as orc
from tests.test_gpu_experts import BF16, F32, check_combine, check_quantize, check_routing, check_scaled, ints, normal, ok, run_routing, small_codes, small_scales, uneven, values, workspace

pytestmark = pytest.mark.gpu


def long_tailed(r, most):
    return int(np.clip(np.exp(r.uniform(0, np.log(most + 1))), 1, most))


@pytest.mark.parametrize("seed", range(24))
def test_drawn_routing(seed):
    r = np.random.default_rng(seed)
    for _ in range(4):
        tokens, experts = long_tailed(r, 1500), long_tailed(r, 512)
        groups = int(r.choice([g for g in range(1, 33) if experts % g == 0]))
        top_groups = int(r.integers(1, groups + 1))
        k = int(r.integers(1, min(32, experts // groups * top_groups) + 1))
        dtype = BF16 if r.integers(2) else F32
        logits = normal((tokens, experts + int(r.integers(0, 9))), dtype, seed, float(r.choice([0.01, 1.0, 20.0])))[:, :experts]
        if r.integers(3) == 0:
            logits = (logits * 4).round().div(4)          # ties
        bias = normal((experts,), F32, seed + 1, float(r.choice([0.01, 1.0]))) if r.integers(2) else None
        positions = ints(r.integers(-1, 5, tokens)) if r.integers(2) else None
        check_routing(logits, k, str(r.choice(["softmax", "sigmoid"])), bias, groups, top_groups, bool(r.integers(2)), float(r.choice([1.0, 0.1, 16.0])), positions)


@pytest.mark.parametrize("tokens", [1, 2, 7, 8, 9, 15, 16, 17, 63, 64, 65, 112, 113, 120, 121, 127, 128, 129, 143, 144, 145])
def test_routing_of_few_tokens(tokens):
    """Both sides of the border between one launch and two, and tokens that the CTAs of a cluster do not share evenly."""
    for experts, groups, top_groups, k in ((5, 1, 1, 3), (512, 1, 1, 8), (96, 3, 2, 32)):
        positions = ints(np.where(np.arange(tokens) % 5 == 3, -1, np.arange(tokens)))
        check_routing(normal((tokens, experts), F32, tokens, 1.5), k, "sigmoid", normal((experts,), F32, 1, 0.1), groups, top_groups, True, 1.0, positions)
        check_routing(normal((1, experts), F32, 3).expand(tokens, experts).contiguous(), k, "softmax", None, groups, top_groups)   # all tokens alike


@pytest.mark.parametrize("scoring", ["sigmoid", "softmax"])
def test_groups_whose_sums_32_bits_cannot_tell_apart(scoring):
    """Biases that cancel in a group's sum, equal groups, groups a step of fp32 apart, experts and whole groups that are switched off."""
    e, groups, per = 64, 8, 8
    g = torch.Generator("cuda").manual_seed(3)
    logits = torch.randn((400, e), generator=g, device="cuda") * 0.01
    bias = torch.zeros(e, device="cuda")
    bias[0::per], bias[1::per], bias[2::per] = 50.0, -49.99, -49.98   # sums near 0 of values near 50, rounded to 2^-18
    for i in range(3, per):
        bias[i::per] = -60.0
    for top_groups in (1, 4, 7):
        check_routing(logits, 4, scoring, bias, groups, top_groups)
    same = logits.view(400, groups, per)[:, :1].expand(400, groups, per).reshape(400, e).contiguous()
    for top_groups in (1, 3, 7):
        check_routing(same, 5, scoring, None, groups, top_groups)   # equal groups: the first ones
        check_routing(same, 5, scoring, torch.zeros(e, device="cuda"), groups, top_groups)
    step = same.view(torch.int32) + torch.randint(-1, 2, same.shape, generator=g, device="cuda", dtype=torch.int32)
    check_routing(step.view(torch.float32), 6, scoring, None, groups, 4, True, 2.0)
    off = torch.zeros(e, device="cuda")
    off[8:16], off[17], off[33:40] = -float("inf"), -float("inf"), -float("inf")   # a group, one expert, all but one of a group
    off[48] = float("inf")
    check_routing(step.view(torch.float32), 6, scoring, off, groups, 3)
    check_routing(logits, 6, scoring, off, groups, 7)


@pytest.mark.parametrize("seed", range(16))
def test_drawn_quantize(seed):
    r = np.random.default_rng(100 + seed)
    for _ in range(4):
        dtype, gated = BF16 if r.integers(2) else F32, bool(r.integers(2))
        rows, cols, shift = long_tailed(r, 900), 16 * long_tailed(r, 150), int(r.choice([0, 0, 1, 2, 8]))
        x = normal((rows, cols * (2 if gated else 1) + shift + int(r.integers(0, 9))), dtype, seed, float(r.choice([1e-3, 1.0, 50.0])))
        x = x[:, shift: shift + cols * (2 if gated else 1)]
        if not gated and r.integers(3) == 0:
            check_quantize(x, block_rows=128, pad=16 * int(r.integers(0, 3)))
        else:
            check_quantize(x, gated, int(r.choice([0, 1, 2, 7])), pad=16 * int(r.integers(0, 3)), seed=seed, some_outside=bool(r.integers(2)))


@pytest.mark.parametrize("dtype,std", [(BF16, 1.0), (F32, 1.0), (F32, 10.0), (BF16, 30.0), (F32, 1e-3)])
def test_gated_codes_are_the_nearest(dtype, std):
    """Codes against the quotients in 64 bits by the kernel's own scales, all of them; scales: of the largest, rounded once, but
    where a value of less than 2^-15 below it stands in for it (which takes two such in 16 neighbours: one block in ten thousand)."""
    rows, cols = 3000, 1408
    x = normal((rows, 2 * cols), dtype, 11, std)
    codes, scales = torch.zeros((rows, cols), dtype=torch.uint8, device="cuda"), torch.zeros((rows, cols // 128), device="cuda")
    dvm.launch(dvm.encode_quantize(x, codes, scales, gated=True), [x, codes, scales])
    ok()
    z, u = x.double()[:, :cols], x.double()[:, cols:]
    v = torch.where(z < -87, 0.0, z / (1 + (-z).exp())) * u
    largest = (v.abs().view(rows, -1, 128).amax(2) / 448).clamp(min=2.0 ** -126)
    assert bool(((scales.double() - largest).abs() <= largest * 2.0 ** -15).all())
    assert float((scales != largest.float()).float().mean()) <= 1e-3
    q = (v.view(rows, -1, 128) / scales.double()[..., None]).view(rows, cols)
    table = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    m = q.abs().clamp(max=448.0)
    hi = torch.searchsorted(table, m).clamp(1, 126)
    up = m - table[hi - 1] - (table[hi] - m)
    at = torch.where((up > 0) | ((up == 0) & (hi % 2 == 0)), hi, hi - 1)
    assert torch.equal(codes & 0x7f, at.to(torch.uint8))
    assert bool((((codes >> 7) == 1) == (q < 0))[at > 0].all())


@pytest.mark.parametrize("seed", range(32))
def test_drawn_scaled(seed):
    r = np.random.default_rng(200 + seed)
    for _ in range(3):
        groups = long_tailed(r, 200) if r.integers(3) else 1
        rows, n, k = long_tailed(r, 4000), long_tailed(r, 1200), 16 * long_tailed(r, 120)
        check_scaled(uneven(rows, groups, seed) if groups > 1 else [rows], n, k, BF16 if r.integers(2) else F32, exact=bool(r.integers(4)), pad=int(r.choice([0, 0, 1, 4, 8])),
                     grouped=groups > 1 or bool(r.integers(2)), behind=int(r.choice([0, 1, 40])), seed=seed, x_pad=16 * int(r.integers(0, 3)))


@pytest.mark.parametrize("seed", range(16))
def test_drawn_combine(seed):
    r = np.random.default_rng(300 + seed)
    for _ in range(4):
        tokens, k, cols = long_tailed(r, 600), int(r.integers(1, 33)), long_tailed(r, 2500)
        check_combine(tokens, k, long_tailed(r, 2000), cols, BF16 if r.integers(2) else F32, bool(r.integers(2)), int(r.choice([0, 1, 8])), int(r.choice([0, 0, 1, 4])), seed=seed)


@pytest.mark.parametrize("rows,groups,n,tile", [
    (1, 1, 4096, 16), (12, 1, 40000, 16), (13, 1, 40000, 128), (13, 1, 18944, 16), (32, 1, 9472, 16), (32, 1, 9473, 64), (32, 1, 18944, 64), (32, 1, 18945, 128),
    (33, 1, 18944, 64), (33, 1, 18945, 128), (128, 1, 9472, 64), (129, 1, 9472, 128), (128, 1, 9473, 128), (1000, 100, 128, 16), (1300, 100, 128, 16), (3300, 100, 128, 64), (1300, 100, 300, 128)])
def test_which_kernel_takes_it(rows, groups, n, tile):
    """On both sides of the rule's borders: mean rows of a group, and tiles against the SMs."""
    k = 144
    check_scaled(uneven(rows, groups, 3) if groups > 1 else [rows], n, k, grouped=groups > 1, behind=0, exact=True)
    assert dvm.last_scaled_matmul_tile() == tile


@pytest.mark.parametrize("dtype,n,pad,shift", [(BF16, 256, 0, 0), (BF16, 255, 0, 0), (BF16, 264, 4, 0), (BF16, 512, 0, 1), (F32, 256, 0, 0), (F32, 257, 2, 0), (F32, 100, 0, 3), (F32, 1000, 1, 1), (BF16, 40, 8, 4)])
@pytest.mark.parametrize("counts", [[9600], [1, 127, 128, 129, 700, 9000], [31, 33, 0, 1, 64, 900, 9000]])
def test_many_rows_into_any_layout(dtype, n, pad, shift, counts):
    """The kernel for many rows with results that its copies out cannot take (offsets, strides) and with groups that end inside a tile:
    nothing is written beside them."""
    k, rows = 400, sum(counts) + 5
    x, xs, groups = small_codes((rows, k), 1), small_scales((rows, 4), 2), len(counts)
    w, ws = small_codes((groups, n, k), 3), small_scales((groups, -(-n // 128), 4), 4)
    whole = torch.full((rows + 2, n + pad + 16), 7.0, dtype=dtype, device="cuda")
    out = whole.as_strided((rows, n), (n + pad + 16, 1), n + pad + 16 + shift)
    first = np.concatenate([[0], np.cumsum(counts)])
    code = dvm.encode_scaled_matmul(x, xs, w, ws, out, ints(first))
    dvm.launch(code, [x, xs, w, ws, ints(first), out, workspace(code)])
    ok()
    assert dvm.last_scaled_matmul_tile() == 128
    X, W = values(x, xs, 1), values(w, ws, 128)
    want = torch.full(whole.shape, 7.0, dtype=torch.float64, device="cuda")
    for g in range(groups):
        want.as_strided((rows, n), out.stride(), out.storage_offset())[first[g]: first[g + 1]] = (X[first[g]: first[g + 1]] @ W[g].T).to(dtype).double()
    assert torch.equal(whole.double(), want)


def test_offsets_past_32_bits():
    """300000 rows of 8192 values, written by the rows of a permutation, multiplied (both kernels) and added up: the rows on both
    sides of what 32 bits count are those of a call of these rows alone."""
    rows, cols = 300000, 8192
    g = torch.Generator("cuda").manual_seed(5)
    x = torch.empty((rows, cols), dtype=BF16, device="cuda").normal_(generator=g)
    codes, scales = torch.zeros((rows, cols), dtype=torch.uint8, device="cuda"), torch.zeros((rows, 64), device="cuda")
    places = torch.randperm(rows, generator=g, device="cuda").int().reshape(rows, 1)
    dvm.launch(dvm.encode_quantize(x, codes, scales, places), [x, places, codes, scales])
    ok()
    some = [0, 1, 2 ** 31 // cols - 1, 2 ** 31 // cols, 2 ** 31 // cols + 1, 2 ** 30 // cols, rows - 1]
    pick = torch.tensor(some, device="cuda")
    few, at = x[pick].contiguous(), places[pick, 0].long()
    c, s = torch.zeros((len(some), cols), dtype=torch.uint8, device="cuda"), torch.zeros((len(some), 64), device="cuda")
    dvm.launch(dvm.encode_quantize(few, c, s), [few, c, s])
    ok()
    assert torch.equal(codes[at], c) and torch.equal(scales[at], s)
    inverse = torch.empty(rows, dtype=torch.long, device="cuda")
    inverse[places[:, 0].long()] = torch.arange(rows, device="cuda")
    source = x[inverse[pick]].contiguous()
    dvm.launch(dvm.encode_quantize(source, c, s), [source, c, s])
    ok()
    assert torch.equal(codes[pick], c) and torch.equal(scales[pick], s)

    # the product: x itself is the place of the result
    n = cols
    w, ws = small_codes((2, n, cols), 3), small_scales((2, 64, 64), 4)
    starts = ints([0, 150000, rows - 1])
    last = x[-1].clone()
    code = dvm.encode_scaled_matmul(codes.view(torch.float8_e4m3fn), scales, w, ws, x, starts)
    dvm.launch(code, [codes, scales, w, ws, starts, x, workspace(code)])
    ok()
    assert dvm.last_scaled_matmul_tile() == 128
    assert torch.equal(x[-1], last)
    for r in some[:-1] + [rows - 2]:
        want = values(codes[r: r + 1].view(torch.float8_e4m3fn), scales[r: r + 1], 1) @ values(w[int(r >= 150000)], ws[int(r >= 150000)], 128).T
        mag = values(codes[r: r + 1].view(torch.float8_e4m3fn), scales[r: r + 1], 1).abs() @ values(w[int(r >= 150000)], ws[int(r >= 150000)], 128).abs().T
        bound = orc.scaled_bound(want.cpu().numpy(), mag.cpu().numpy(), 64, BF16)
        assert ((x[r: r + 1].double() - want).abs().cpu().numpy() <= bound).all(), r

    # combine: rows far down, and a result as long
    y, out = x, torch.full((rows, cols), 7.0, dtype=BF16, device="cuda")
    weights = torch.ones((rows, 1), device="cuda")
    dvm.launch(dvm.encode_combine(y, places, weights, out), [y, places, weights, out])
    ok()
    assert torch.equal(out[pick], y[at]) and torch.equal(out[-5000:], y[places[-5000:, 0].long()])


def test_offsets_past_32_bits_in_the_weights():
    """300 weights of 1024 x 8192, the last with a row: 2.5e9 codes."""
    groups, n, k = 300, 1024, 8192
    w, ws = torch.zeros((groups, n, k), dtype=torch.uint8, device="cuda"), torch.zeros((groups, 8, 64), device="cuda")
    for g in (0, 255, 256, 299):
        w[g], ws[g] = small_codes((n, k), g).view(torch.uint8), small_scales((8, 64), g)
    for each in (1, 3000):                       # few rows, many rows
        first = np.zeros(groups + 1, dtype=np.int64)
        for g in (0, 255, 256, 299):
            first[g + 1:] += each
        rows = int(first[-1])
        x, xs = small_codes((rows, k), 7), small_scales((rows, 64), 8)
        out = torch.full((rows, n), 7.0, device="cuda")
        code = dvm.encode_scaled_matmul(x, xs, w.view(torch.float8_e4m3fn), ws, out, ints(first))
        dvm.launch(code, [x, xs, w, ws, ints(first), out, workspace(code)])
        ok()
        for g in (0, 255, 256, 299):
            a, b = int(first[g]), int(first[g + 1])
            want = values(x[a:b], xs[a:b], 1) @ values(w[g].view(torch.float8_e4m3fn), ws[g], 128).T
            assert torch.equal(out[a:b].double(), want), g


def test_a_dense_product_right_behind_what_writes_its_weight():
    """The weight's codes are written by the launch just before, other ones each time: none of the last ones are read."""
    n, k = 11008, 1024
    x, xs = small_codes((3, k), 1), small_scales((3, 8), 2)
    values_of = [normal((n, k), BF16, seed) for seed in (3, 4)]
    w, ws = torch.zeros((n, k), dtype=torch.uint8, device="cuda"), torch.zeros((n // 128, 8), device="cuda")
    out = [torch.empty((3, n), device="cuda") for _ in range(40)]
    quantize = dvm.encode_quantize(values_of[0], w, ws, block_rows=128)
    product = dvm.encode_scaled_matmul(x, xs, w[None], ws[None], out[0])
    work, want = workspace(product), []
    for v in values_of:
        dvm.launch(quantize, [v, w, ws])
        torch.cuda.synchronize()
        dvm.launch(product, [x, xs, w, ws, out[0], work])
        ok()
        want.append(out[0].clone())
    assert not torch.equal(want[0], want[1])
    for i in range(40):
        dvm.launch(quantize, [values_of[i % 2], w, ws])
        dvm.launch(product, [x, xs, w, ws, out[i], work])
    ok()
    for i in range(40):
        assert torch.equal(out[i], want[i % 2]), i


def test_routing_on_two_streams_at_once():
    """Clusters of two calls side by side, and calls of one launch between calls of two."""
    a, b = normal((128, 256), F32, 1, 1.5), normal((300, 512), F32, 2, 1.5)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()

    def call(logits):
        t, e = logits.shape
        out = [torch.full((t, 8), 77, dtype=dt, device="cuda") for dt in (torch.int32, F32, torch.int32)] + [ints(np.full(e + 1, 77))]
        code = dvm.encode_routing(logits, 8)
        return code, [logits] + out + [workspace(code)]

    calls = [(call(a), call(b), call(a[: i + 1])) for i in range(30)]
    torch.cuda.synchronize()                                        # (the tensors are there before the other streams use them)
    for x, y, z in calls:
        dvm.launch(*x, one)
        dvm.launch(*y, two)
        dvm.launch(*z, two)
    ok()
    of_a, of_b = run_routing(a, 8), run_routing(b, 8)
    ok()
    for i, (x, y, z) in enumerate(calls):
        assert all(torch.equal(p, q) for p, q in zip(x[1][1:5] + y[1][1:5], of_a + of_b)), i
        assert all(torch.equal(p, q[: i + 1]) for p, q in zip(z[1][1:3], of_a[:2])), i
