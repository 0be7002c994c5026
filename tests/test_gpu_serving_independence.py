"""A request's answer does not depend, in any bit, on what other rows hold: rows behind the last request (padding that nobody
wrote) and, for prompts, the queries and keys of other requests."""
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests.test_gpu_serving import BF16, F32, Batch, ints, normal, ok

pytestmark = pytest.mark.gpu

CASES = [(4, 2, 64, 16, 0, 0), (5, 1, 96, 8, 0, 0), (3, 3, 128, 64, 40, 3), (16, 1, 128, 16, 0, 0), (40, 2, 64, 16, 100, 1)]


def answer(b, max_q, window, sinks):
    out = torch.full(b.q.shape, 7.0, dtype=F32, device="cuda")
    b.launch(b.code(out, scale=0.125, window=window, sinks=sinks, max_q=max_q), out)
    ok()
    return out


@pytest.mark.parametrize("hq,hk,dim,page,window,sinks", CASES)
@pytest.mark.parametrize("fresh", [1, 7, 45])
def test_rows_behind_the_last_request(hq, hk, dim, page, window, sinks, fresh):
    b = Batch([300, 200], [fresh, fresh], hq, hk, dim, page, pad=70, seed=fresh, std=0.5)
    rows, kernel = 2 * fresh, "single" if fresh == 1 and hq // hk <= 16 else "prompt"
    b.q[rows:] = 0
    want = answer(b, fresh, window, sinks)
    assert dvm.last_attention_kernel() == kernel
    for fill in (normal(b.q[rows:].shape, BF16, 5, 40.0), float("nan"), float("inf"), -float("inf"), torch.finfo(BF16).max):
        b.q[rows:] = fill
        assert torch.equal(answer(b, fresh, window, sinks), want)


@pytest.mark.parametrize("hq,hk,dim,page,window,sinks", CASES)
def test_prompts_of_other_requests(hq, hk, dim, page, window, sinks):
    lengths, fresh = [300, 411, 90, 64], [45, 130, 7, 64]
    b = Batch(lengths, fresh, hq, hk, dim, page, seed=3, std=0.5)
    want = answer(b, 130, window, sinks)
    at = 0
    for i, f in enumerate(fresh):
        mine, rest = slice(at, at + f), [r for r in range(b.q.shape[0]) if not at <= r < at + f]
        q, table, starts, lens = b.q.clone(), b.table.clone(), b.starts.clone(), list(b.lengths)
        for fill in (normal(q[rest].shape, BF16, 6, 40.0), float("nan")):
            b.q[rest] = fill
            assert torch.equal(answer(b, 130, window, sinks)[mine], want[mine])
        # the request on its own
        b.q, b.table, b.starts, b.lengths = q[mine].contiguous(), table[i:i + 1].contiguous(), ints([0, f]), [lens[i]]
        assert torch.equal(answer(b, 130, window, sinks), want[mine])
        b.q, b.table, b.starts, b.lengths = q, table, starts, lens
        at += f


def test_the_same_launch_again():
    for fresh, max_q in (([1, 1, 1], 1), ([60, 33, 7], 60)):
        b = Batch([2000, 90, 500], fresh, 8, 2, 128, 16, seed=6)
        want = answer(b, max_q, 0, 0)
        assert all(torch.equal(answer(b, max_q, 0, 0), want) for _ in range(20))
