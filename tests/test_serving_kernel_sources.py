"""What the compiler made of the serving kernels (`-Xptxas -v`), and the polynomial of the prompts' weights in numpy."""
import os
import re

import numpy as np
import pytest

from tests.test_kernel_resources import CSRC, NVCC, _resources


@pytest.mark.skipif(not os.path.exists(NVCC), reason="nvcc not found")
@pytest.mark.parametrize("source,kernel,least,most", [
    ("dvm_attention_prompt.cu", "prompt_kernel", 168, 168),   # 384 threads: what setmaxnreg deals out by role is counted from this
    ("dvm_attention_single.cu", "single_kernel", 1, 200),     # two CTAs of 160 threads per SM
    ("dvm_attention_single.cu", "join_kernel", 1, 64),
    ("dvm_attention.cu", "plain_kernel", 1, 64),
    ("dvm_paging.cu", "paging_kernel", 1, 64),
])
def test_attention_and_paging_do_not_spill(source, kernel, least, most):
    res = {k: v for k, v in _resources(source).items() if kernel in k}
    assert res, kernel
    for name, (regs, stack, st, ld) in res.items():
        assert stack == 0 and st == 0 and ld == 0, (name, regs, stack, st, ld)
        assert least <= regs <= most, (name, regs)


@pytest.mark.skipif(not os.path.exists(NVCC), reason="nvcc not found")
def test_rotary_does_not_spill():
    res = {k: v for k, v in _resources("dvm_rotary.cu").items() if "rotary_kernel" in k}
    assert len(res) == 28                                      # 4 pairs of types: 3 widths x 2 pairings, and the kernel for other layouts
    for name, (regs, stack, st, ld) in res.items():
        assert stack == 0 and st == 0 and ld == 0, (name, regs, stack, st, ld)
        assert regs <= (128 if "Li0E" in name else 85), (name, regs)   # two, three CTAs of 256 threads per SM


def polynomial():
    text = open(os.path.join(CSRC, "dvm_attention_prompt.cu")).read()
    body = text[text.index("float2 ex2_by_polynomial("):]
    body = body[:body.index("\n}\n")]
    return [np.float32(x) for x in re.findall(r"make_float2\((\d\.\d+)f, ", body)] + [np.float32(1)]


def by_polynomial(x):
    """The device's steps: every operation rounds to fp32 once (a product and sum of fp32 in 64 bits, then to fp32)."""
    c = polynomial()
    x = np.where(np.isnan(x), np.float32(-127), np.maximum(x, np.float32(-127))).astype(np.float32)   # (fmaxf)
    t = x + np.float32(12582912)
    r = x - (t - np.float32(12582912))
    p = np.full_like(x, c[0])
    for k in c[1:]:
        p = (p.astype(np.float64) * r + np.float64(k)).astype(np.float32)
    return (p.view(np.int32) + (t.view(np.int32) << np.int32(23))).view(np.float32)


def test_exponentials_by_polynomial():
    c = polynomial()
    assert len(c) == 6 and c[-1] == 1
    # the polynomial itself: 9.15e-8 (Remez exchange); its coefficients rounded to fp32 add, of a value of at least 2^-1/2, half a
    # step of each times its power of r: (2^-25 / 2 + 2^-27 / 4 + 2^-29 / 8 + ...) sqrt(2) < 2.42e-8
    r = np.linspace(-0.5, 0.5, 200001)
    assert np.abs(np.polyval(np.array(c, np.float64), r) / np.exp2(r) - 1).max() < 1.16e-7
    # as evaluated: the last step rounds once (2^-24 of the value), those before by the same half steps as above (below 2^-25)
    rng = np.random.default_rng(1)
    x = np.concatenate([np.linspace(-126, 127.4, 1000001), rng.uniform(-126, 9, 1000000), np.arange(-252, 255) / 2]).astype(np.float32)
    got = by_polynomial(x).astype(np.float64)
    assert np.abs(got / np.exp2(x.astype(np.float64)) - 1).max() < 1.16e-7 + 1.5 * 2.0 ** -24
    n = np.arange(-126, 128).astype(np.float32)
    assert np.array_equal(by_polynomial(n), np.ldexp(np.float32(1), n.astype(int)))        # whole numbers: exact
    low = np.array([-127, -128, -1e4, -3e38, -np.inf], np.float32)
    assert (by_polynomial(low) == 0).all()                     # hidden tokens: exactly nothing
    near = np.linspace(-127, -126, 10001).astype(np.float32)   # below the normal numbers: between nothing and 2^-126
    assert ((by_polynomial(near) >= 0) & (by_polynomial(near) <= np.float32(2.0 ** -126))).all()
