"""Rows that are done again without tensor cores (an infinite value in a tile that some of them see and others do not) while the
rest of their block's warps wait: on a long cache that takes longer than any wait's limit, and still answers."""
import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests.test_gpu_serving import BF16, F32, I32, ints

pytestmark = pytest.mark.gpu


LONG = 64 * 2400   # 2.5 s


def run(length, rows=40, page=64, dim=8, heads=2):
    """Queries of zero (weights of 1) over a cache whose table names the same few pages again and again; the last page is its own:
    there a token of value 1 + c in column c, and behind most rows an infinity in column 3 of head 0.  Milliseconds on the device."""
    assert length % page == 0
    k = torch.ones((40, page, heads, dim), dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    for c in range(dim):
        v[39, c, :, c] = 1.0 + c
    v[39, page - 20, 0, 3] = float("inf")
    table = np.random.default_rng(1).integers(0, 39, (1, length // page))
    table[0, -1] = 39
    q = torch.zeros((rows, heads, dim), dtype=BF16, device="cuda")
    out = torch.full((rows, heads, dim), 7.0, dtype=F32, device="cuda")
    table = ints(table)
    code = dvm.encode_attention(q=q, k_cache=k, v_cache=v, table=table, out=out, scale=1.0, max_q=rows)
    at = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    args = [q, k, v, table, ints([0, rows]), ints([length]), out, torch.empty(16, dtype=torch.uint8, device="cuda")]
    at[0].record()
    dvm.launch(code, args)
    at[1].record()
    assert dvm.last_device_status() == 0
    assert dvm.last_attention_kernel() == "prompt"
    got = out.cpu().double().numpy()
    for t in range(rows):
        p = length - rows + t
        want = np.tile((1.0 + np.arange(dim)) / (p + 1), (heads, 1))
        if p >= length - 20:
            want[0, 3] = np.inf
        with np.errstate(invalid="ignore"):
            assert ((got[t] == want) | (np.abs(got[t] - want) <= 2.0 ** -21 * want)).all(), (t, got[t], want)
    return at[0].elapsed_time(at[1])


def test_rows_done_again():
    run(640)
    run(8192)


def test_rows_done_again_for_longer_than_a_wait_may_last():
    """More than the 2 s that a wait gives work that shows no sign of going on."""
    assert run(LONG) > 2200
