"""The operators of a layer of experts where their numbers are at the ends of what fp32 holds, and at sizes near 2^31."""
import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests import experts_oracle as orc
from tests.experts_oracle import f64
from tests.test_gpu_experts import F32, check_routing, ints, normal, ok, run_routing

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------ routing

def check_renormalised(logits, top_k, scoring, bias=None, groups=1, top_groups=1, factor=1.0):
    """As check_routing, the weights by logarithms of the scores, of finite logits: quotients of the scores themselves are 0 / 0 in 64 bits
    too from logits of -746 down (exp(746) passes 2^1024)."""
    ids, weights, places, starts = (x.cpu().numpy() for x in run_routing(logits, top_k, scoring, bias, groups, top_groups, True, factor))
    ok()
    want = orc.routing(f64(logits), top_k, scoring, None if bias is None else f64(bias), groups, top_groups, False, 1.0, None)
    assert np.array_equal(ids, want[0]) and np.array_equal(places, want[2]) and np.array_equal(starts, want[3])
    chosen = np.take_along_axis(f64(logits), ids.astype(np.int64), 1)
    log_s = chosen if scoring == "softmax" else -np.logaddexp(0.0, -chosen)    # (a softmax's common denominator left out)
    w = np.exp(log_s - np.logaddexp.reduce(log_s, 1, keepdims=True)) * factor
    assert (np.abs(weights - w) <= w * orc.weights_bound(logits.shape[1]) + 2.0 ** -126).all()


@pytest.mark.parametrize("tokens", [5, 200])
@pytest.mark.parametrize("top_k", [1, 4])
def test_renormalised_weights_of_scores_below_fp32(tokens, top_k):
    """The definition's quotients are ordinary numbers however small the scores are.  (weights_bound: differences of the chosen logits are
    below 30 here too.)"""
    e = 64
    base = normal((tokens, e), F32, 1, 3.0)
    for shift in (-60.0, -85.0, -88.0, -100.0, -120.0, -400.0, -650.0):
        for groups, top_groups in ((1, 1), (8, 3)):
            check_renormalised(base + shift, top_k, "sigmoid", None, groups, top_groups, 2.5)
        check_renormalised(base + shift, top_k, "sigmoid", normal((e,), F32, 2, 0.3))
    # a bias that chooses experts far below the top
    for below in (60.0, 90.0, 95.0, 104.0, 120.0, 400.0, 650.0):
        logits, bias = base.clone(), torch.zeros(e, device="cuda")
        bias[8:16] = 2.0
        logits[:, 8:16] -= below
        check_renormalised(logits, top_k, "softmax", bias)
        check_renormalised(logits, top_k, "softmax", bias, 8, 2, 0.5)
        check_renormalised(logits - 300.0, top_k, "sigmoid", bias, 8, 2)
    # one chosen score of ordinary size beside ones that are not
    logits = base - 130.0
    logits[:, 3] = 1.0
    check_renormalised(logits, top_k, "sigmoid")
    check_renormalised(logits, top_k, "softmax")
    logits[:, 3] = -50.0
    check_renormalised(logits, top_k, "sigmoid")


def test_renormalised_weights_of_values_that_are_not_finite():
    """A NaN or +inf logit under softmax makes the weights NaN, whatever is chosen; so do chosen scores that are all zero, those of -inf."""
    e, inf, nan = 64, float("inf"), float("nan")
    base, zeros, high = normal((40, e), F32, 5), torch.zeros(e, device="cuda"), torch.zeros(e, device="cuda")
    high[10:20] = 3.0
    for bad in (nan, inf, -inf):
        x = base.clone()
        x[1, 5], x[3, :], x[7, 12:], x[9, 10:20] = bad, bad, bad, bad
        for bias in (zeros, high):
            check_routing(x, 6, "softmax", bias, renormalise=True)
            check_routing(x, 6, "sigmoid", bias, renormalise=True)
        check_routing(x, 6, "softmax", renormalise=True)
        if bad != bad:
            continue
        check_routing(x, 6, "sigmoid", renormalise=True)
        check_routing(x, 6, "sigmoid", None, 8, 5, True)
    # the lowest finite logits are numbers like any others: alike ones share alike (exact arithmetic: 64 bits have 0 / 0 here)
    x = base.clone()
    x[::2] = torch.finfo(F32).min
    for positions in (None, ints(np.arange(40) % 3 - 1)):
        _, weights, _, _ = run_routing(x, 4, "sigmoid", renormalise=True, positions=positions)
        ok()
        takes_part = torch.ones(40, dtype=torch.bool, device="cuda") if positions is None else positions >= 0
        assert bool((weights[::2] == torch.where(takes_part, 0.25, 0.0)[::2, None]).all())


def test_softmax_without_a_number():
    """All of a token's scores are NaN: groups, and experts with a bias, are taken by index, experts without one by their logits."""
    e, inf, nan = 96, float("inf"), float("nan")
    x = normal((150, e), F32, 7)
    x[::3, 40], x[1::3, 90], x[2::6, 5], x[5::6] = nan, inf, nan, -inf
    high = normal((e,), F32, 8)
    for groups, top_groups in ((1, 1), (8, 5)):
        for renormalise in (False, True):
            check_routing(x, 6, "softmax", None, groups, top_groups, renormalise)
            check_routing(x, 6, "softmax", high, groups, top_groups, renormalise)
    ids, weights, _, _ = run_routing(x, 6, "softmax", high)
    ok()
    assert bool(weights.isnan().all()) and bool((ids == torch.arange(6, device="cuda")).all())
    ids, _, _, _ = run_routing(x[:1], 6, "softmax")
    assert torch.equal(ids[0].long(), x[0].nan_to_num(-inf).sort(descending=True, stable=True)[1][:6])


# ------------------------------------------------------------------------------------------------------ sizes near 2^31

@pytest.mark.parametrize("cols", [2 ** 31 - 1, 2 ** 31 - 61])
def test_combine_of_as_many_columns_as_a_size_can_name(cols):
    """Odd numbers of columns, one to a thread: the last ones, and those on both sides of the last whole piece of 64, are written too."""
    torch.cuda.empty_cache()
    y = torch.empty((1, cols), dtype=torch.bfloat16, device="cuda").fill_(3.0)
    out = torch.full((1, cols), 7.0, dtype=torch.bfloat16, device="cuda")
    places, weights = ints([[0]]), torch.ones((1, 1), device="cuda")
    dvm.launch(dvm.encode_combine(y, places, weights, out), [y, places, weights, out])
    ok()
    assert bool((out == 3.0).all())
    del y, out
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------------ gated codes

def spread_values(shape, lo, hi, dtype, seed, signed=True):
    """Magnitudes 2^lo .. 2^hi, evenly in their logarithms."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.exp2(torch.rand(shape, generator=g, device="cuda") * (hi - lo) + lo)
    return (v * torch.sign(torch.randn(shape, generator=g, device="cuda")) if signed else v).to(dtype)


def check_gated(z, u):
    """Codes nearest to the quotients in 64 bits by the kernel's own scales, all of them; scales of the largest value, or of one less than
    2^-15 below it.  Values of 2^128 and more are infinities (as near to 2^128 as the kernel's fp32 may be off, 2^-16, they may be or not)."""
    rows, cols = z.shape
    x = torch.cat([z, u], 1)
    codes, scales = torch.full((rows, cols), 0x11, dtype=torch.uint8, device="cuda"), torch.full((rows, -(-cols // 128)), 7.0, device="cuda")
    dvm.launch(dvm.encode_quantize(x, codes, scales, gated=True), [x, codes, scales])
    ok()
    z, u = z.double(), u.double()
    v = torch.where(z < -87.336544, 0.0, z / (1 + (-z).exp())) * u          # (126 ln 2)
    v = torch.nn.functional.pad(v, (0, -cols % 128)).view(rows, -1, 128)
    largest = (v.abs().amax(2) / 448).clamp(min=2.0 ** -126)
    top = largest * 448
    infinite = torch.where((top / 2.0 ** 128 - 1).abs() < 2.0 ** -16, scales.isnan(), top >= 2.0 ** 128)
    assert torch.equal(scales.isnan(), infinite)
    assert bool(((scales.double() - largest).abs() <= largest * 2.0 ** -15)[~infinite].all())
    q = torch.where(infinite[..., None], 0.0, v / scales.double()[..., None]).view(rows, -1)[:, :cols]
    want = torch.from_numpy(orc.encode(q.cpu().numpy())).cuda()
    assert torch.equal(codes & 0x7f, want & 0x7f)
    assert bool(((codes >> 7) == (q < 0))[(want & 0x7f) > 0].all())


@pytest.mark.parametrize("dtype", [F32, torch.bfloat16])
@pytest.mark.parametrize("z_lo,z_hi,u_lo,u_hi", [
    (-149, -124, 90, 127),      # gates among fp32's subnormals, values that are not
    (-149, -100, 60, 127), (-126, 6, 0, 20),
    (-1, 1, -149, -105),        # the other way round
    (-20, 3, -130, -118),       # blocks of the least scale and a little above
    (-10, 6, -149, -100), (-149, 6, -149, 100), (3, 6.4, -149, -120), (3, 6.4, 60, 125)])
def test_gated_codes_of_small_and_large_factors(dtype, z_lo, z_hi, u_lo, u_hi):
    for seed, n in ((1, 3000), (2, 500)):
        z, u = spread_values((n, 272), z_lo, z_hi, dtype, seed), spread_values((n, 272), u_lo, u_hi, dtype, seed + 10)
        check_gated(z, u)
        check_gated(-z.abs(), u)
        check_gated(z.abs(), u)


def test_gated_where_silu_becomes_zero():
    """At one place (-126 ln 2, -87.3365) for what the scale is of and for the codes, whatever stands beside it; values that count are those
    before large ones.  In fp32 the place is off by 2^-16 at most: half a step of the exponent 126 (2^-18) and log2 e's rounding (2^-19), the
    exponential's 2 ulp and the sum's rounding (2^-21)."""
    at = -126 * np.log(2.0)
    near = np.float32(at).view(np.int32) + np.arange(-300, 301)                      # steps of fp32 on both sides
    z = np.concatenate([near.astype(np.int32).view(np.float32), np.float32([-86.9, -87.0, -87.1, -87.25, -87.3, -87.33, -87.34, -87.4, -87.5, -88, -89, -100, -1e4, -3e38])])
    z = torch.tensor(np.repeat(z, 3), device="cuda")
    for u in (3e38, -1e37, 1e30):
        for beside in ((0.0, 0.0), (1.0, 1e-3), (-87.0, 1e38)):                      # the rest of its block: nothing, small, large
            for lane in (0, 5, 127):
                x = torch.zeros((len(z), 256), device="cuda")
                x[:, 1:128:3], x[:, 129::3] = beside
                x[:, lane], x[:, 128 + lane] = z, u
                codes, scales = torch.zeros((len(z), 128), dtype=torch.uint8, device="cuda"), torch.zeros((len(z), 1), device="cuda")
                dvm.launch(dvm.encode_quantize(x, codes, scales, gated=True), [x, codes, scales])
                ok()
                zz, uu = f64(x[:, :128]), f64(x[:, 128:])
                with np.errstate(over="ignore"):
                    full = zz / (1 + np.exp(-zz)) * uu
                # either side of the place, to 2^-16 of it, both answers are one: the whole block's
                got_c, got_s = codes.cpu().numpy(), f64(scales)
                for zero_from in (at - 2.0 ** -16, at + 2.0 ** -16):
                    v = np.where(zz < zero_from, 0.0, full)
                    top = np.maximum(np.abs(v).max(1, keepdims=True) / 448, 2.0 ** -126)
                    right = (np.abs(got_s - top) <= top * 2.0 ** -15) & ((got_c & 0x7f) == (orc.encode(v / got_s) & 0x7f))
                    both = right.all(1) if zero_from < at else both | right.all(1)
                    if zero_from < at:
                        never_zero = right.all(1)
                    else:
                        zero = right.all(1)
                own = zz[:, lane]
                assert both.all()
                assert never_zero[own >= at + 2.0 ** -16].all() and zero[own < at - 2.0 ** -16].all()
