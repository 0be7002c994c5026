"""Every visible token counts, once: queries of zero weigh all visible tokens alike, so a row's answer is the mean of their
values, exactly: weights of 1, sums of whole numbers.  Values are zero but for one token to a column -- the ends of the cache, of tiles,
of ranges, of the window, of the sinks -- so a column is that token's value / n, and one token lost or taken twice anywhere
changes n by more than the roundings (the quotient: a reciprocal and a product, 2^-24 each, and a device division that may be
2 ulp off: 2^-21 covers them) as long as n < 2^20."""
import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests.test_gpu_serving import BF16, F32, Batch, ints, ok

pytestmark = pytest.mark.gpu


def check(lengths, fresh, hq, hk, dim, page, window=0, sinks=0, max_q=1, kernel=None, holes=(), seed=0, dtype=BF16):
    """holes: (request, block) pairs of the table that hold no page."""
    b = Batch(lengths, fresh, hq, hk, dim, page, seed=seed, spare=1, dtype=dtype)
    b.q.zero_()
    b.v.zero_()
    table = b.table.cpu().numpy().copy()
    r = np.random.default_rng(seed)
    marks = []
    for i, n in enumerate(lengths):
        edges = [0, n - 1, n - fresh[i], n - window if window else 0, n - window - fresh[i] + 1 if window else 1, sinks - 1, sinks,
                 63, 64, (n - 1) // 64 * 64, (n - 1) // 64 * 64 - 1, n // 2 // 64 * 64]
        edges += [int(t) + e for t in 64 * r.integers(0, n // 64 + 1, dim // 3) for e in (-1, 0)]   # both sides of tiles and ranges
        edges += [int(t) for t in r.integers(0, n, dim)]
        mine = list(dict.fromkeys(t for t in edges if 0 <= t < n))[:dim]
        for j, t in enumerate(mine):
            b.v[int(table[i, t // page]), t % page, :, j] = float(1 + j % 100)
        marks.append(mine)
    for i, at in holes:
        table[i, at] = -1
    b.table.copy_(ints(table))
    out = torch.full(b.q.shape, 7.0, dtype=F32, device="cuda")
    b.launch(b.code(out, scale=0.125, window=window, sinks=sinks, max_q=max_q), out)
    ok()
    if kernel:
        assert dvm.last_attention_kernel() == kernel
    got = out.cpu().double().numpy()
    row = 0
    for i, n in enumerate(lengths):
        there = np.repeat(table[i] >= 0, page)
        for j in range(fresh[i]):
            p = n - fresh[i] + j
            s = np.arange(len(there))
            seen = there & (s <= p) & ((s > p - window) | (s < sinks) if window else True)
            want = np.zeros(dim)
            for c, t in enumerate(marks[i]):
                if seen[t]:
                    want[c] = (1 + c % 100) / seen.sum()
            bad = np.abs(got[row] - want) > 2.0 ** -21 * np.abs(want)
            assert not bad.any(), (i, j, [(marks[i][c], got[row, h, c], want[c]) for h, c in np.argwhere(bad)[:4]])
            row += 1


@pytest.mark.parametrize("length", [1, 64, 65, 2368, 4737, 9000, 9472, 18945, 32769, 33000, 37000, 37888, 37889, 80000])
@pytest.mark.parametrize("hq,hk", [(1, 1), (7, 1), (8, 8)])
def test_one_single_token(length, hq, hk):
    """Up to 296 parts of one pair; ranges of two tiles and of more."""
    check([length], [1], hq, hk, 64, 64, kernel="single", seed=length)


@pytest.mark.parametrize("lengths", [[37000, 1], [1, 33000], [300, 36000, 300], [18900, 18900], [80000, 5], [9000] * 9])
def test_single_tokens_of_long_and_short_requests(lengths):
    check(lengths, [1] * len(lengths), 3, 1, 64, 16, kernel="single", seed=len(lengths))


@pytest.mark.parametrize("window,sinks", [(1, 0), (4096, 4), (8000, 64), (33000, 1), (100, 3000), (64, 65)])
@pytest.mark.parametrize("lengths", [[40000], [9472, 3000, 70]])
def test_single_tokens_under_a_window(window, sinks, lengths):
    check(lengths, [1] * len(lengths), 4, 1, 128, 16, window, sinks, kernel="single", seed=window)


def test_single_tokens_with_holes():
    check([36000, 4000], [1, 1], 3, 1, 64, 64, kernel="single", holes=[(0, 0), (0, 7), (0, 280), (0, 281), (0, 562), (1, 62)])
    check([36000, 4000], [1, 1], 3, 1, 64, 64, 30000, 100, kernel="single", holes=[(0, 1), (0, 93), (0, 94), (0, 562), (1, 62)])


@pytest.mark.parametrize("lengths,fresh,hq,hk,dim", [([9000], [3], 4, 2, 64), ([40000], [130], 2, 1, 64), ([9472, 700, 64], [1, 700, 64], 4, 2, 128),
                                                     ([20000], [2], 40, 2, 96)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (4096, 4), (65, 64)])
def test_prompts(lengths, fresh, hq, hk, dim, window, sinks):
    check(lengths, fresh, hq, hk, dim, 16, window, sinks, max_q=max(max(fresh), 2), kernel="prompt", seed=dim)


def test_prompts_with_holes():
    check([9000, 500], [200, 300], 4, 2, 64, 16, max_q=300, kernel="prompt", holes=[(0, 0), (0, 5), (0, 300), (0, 555), (1, 3), (1, 30)])
    check([9000, 500], [200, 300], 4, 2, 64, 16, 300, 40, max_q=300, kernel="prompt", holes=[(0, 1), (0, 540), (0, 555), (1, 3), (1, 30)])


def test_without_tensor_cores():
    check([3000, 40], [1, 1], 3, 1, 64, 16, 1000, 4, dtype=F32, kernel="plain")
    check([1200, 40], [30, 40], 2, 1, 64, 16, max_q=40, dtype=F32, kernel="plain")
