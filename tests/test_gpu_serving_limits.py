"""The serving operators at their limits: many requests and heads, many pairs per range, pages of all sizes, the kernel that
takes a call, launches behind other work, in graphs with other nodes, on several streams at once, and other tensors of the
same code."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2603_24239_b200 as dvm
from tests import serving_oracle as orc
from tests.serving_oracle import f64
from tests.test_gpu_serving import BF16, F32, I32, Batch, angles, check_rotary, ints, normal, ok, paging_case, run_paging

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------ sizes

@pytest.mark.parametrize("seed", [0, 1])
def test_paging_with_all_requests_and_rows_that_end_early(seed):
    c, f, free, table, page, rows = paging_case(8192, 90, 3, 16, seed)
    run_paging(c, f, free, table, page, rows)
    run_paging(c, f, free, table, page, rows // 2)     # the rows hold half of the new tokens
    run_paging(c - 40, f - 1, free, table, page, rows)  # lengths below zero count as nothing


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 56), (96, 64), (64, 8), (24, 0), (256, 248)])
def test_rotary_types_pairings_and_parts(dtype, out_dtype, interleaved, dim, rot):
    check_rotary(19, 9, 3, dim, rot, dtype=dtype, out_dtype=out_dtype, interleaved=interleaved, seed=dim)
    check_rotary(19, 9, 3, dim, rot, dtype=dtype, out_dtype=out_dtype, interleaved=interleaved, seed=rot, shift=4, paged=False)


@pytest.mark.parametrize("n,hq,hk,length", [(200, 6, 2, 150), (300, 1, 1, 70), (40, 32, 16, 200), (2, 512, 512, 200), (1, 300, 300, 700), (1, 3, 1, 9000)])
def test_single_tokens_of_more_pairs_than_ranges(n, hq, hk, length):
    r = np.random.default_rng(n)
    lengths = r.integers(0, length + 1, n)
    lengths[-1] = length
    Batch(lengths, [1] * n, hq, hk, 64, 16, seed=n).check(max_q=1, kernel="single")


def test_single_tokens_with_requests_that_have_no_row():
    r = np.random.default_rng(2)
    fresh = (r.random(400) < 0.3).astype(int)
    fresh[0] = fresh[-1] = 0
    b = Batch(r.integers(1, 300, 400), fresh, 4, 1, 64, 16, seed=9)
    b.check(max_q=1, kernel="single")
    b.check(max_q=1, window=64, sinks=4)
    Batch([700], [0], 4, 2, 64, 16, pad=2).check(max_q=1)                          # nothing to answer
    Batch([4000, 50, 2500], [1, 0, 1], 4, 2, 64, 16).check(max_q=1, kernel="single")   # parts to join on both sides of nothing


@pytest.mark.parametrize("length", [1, 63, 64, 65, 127, 128, 129, 2368, 4737, 9472])
def test_one_single_token_of_any_length(length):
    Batch([length], [1], 8, 8, 64, 16, seed=length).check(max_q=1, kernel="single")
    Batch([length], [1], 7, 1, 128, 32, seed=length).check(max_q=1, kernel="single", window=200, sinks=70)


def test_prompts_of_many_requests():
    r = np.random.default_rng(3)
    fresh = r.integers(0, 6, 500)
    fresh[::7] = 0
    fresh[250] = 200
    b = Batch(fresh + r.integers(0, 60, 500), fresh, 4, 2, 64, 16, seed=5)
    b.check(max_q=200, kernel="prompt")
    b.check(max_q=200, window=20, sinks=2, kernel="prompt")


def test_prompts_of_more_blocks_than_the_device_takes_at_a_time():
    Batch([1100, 900, 64], [1000, 900, 64], 24, 8, 64, 64, seed=6).check(max_q=1000, window=96, sinks=1, kernel="prompt")


@pytest.mark.parametrize("page", [8, 16, 64, 128, 1024])
@pytest.mark.parametrize("fresh", [1, 70])
def test_page_sizes(page, fresh):
    Batch([1030, 70, 200], [fresh] * 3, 4, 2, 64, page, seed=page).check(max_q=fresh, window=300, sinks=9, kernel="single" if fresh == 1 else "prompt")


def test_which_kernel_takes_a_call():
    run = lambda kernel, max_q=1, page=16, fresh=1, dim=64, hq=4, hk=2, **kw: Batch([90, 70], [fresh] * 2, hq, hk, dim, page, **kw).check(max_q=max_q, kernel=kernel)  # noqa: E731
    run("single")
    run("single", hq=16, hk=1)
    run("prompt", hq=17, hk=1)              # more heads to a kv head than a range's rows
    run("prompt", max_q=2)
    run("prompt", max_q=20, fresh=20)
    run("plain", dtype=F32)
    run("plain", max_q=20, fresh=20, dtype=F32)
    run("plain", dim=136)
    run("plain", dim=20)


def test_rows_beyond_the_most_of_a_request_are_left():
    Batch([90, 40], [50, 40], 4, 2, 64, 16).check(max_q=8)
    Batch([90, 40], [5, 1], 4, 2, 64, 16).check(max_q=1)


# ------------------------------------------------------------------------------------------------------ order and streams

def test_launches_read_what_the_work_before_them_wrote():
    """Launches may be set up while the work before them ends: they still read only what it has finished."""
    n, page, width = 64, 16, 40
    code = dvm.encode_paging(n, width, page, n, 4096)
    cached, fresh, free = ints(np.zeros(n)), ints(np.zeros(n)), torch.arange(4096, dtype=I32, device="cuda")
    outs = [torch.zeros(m, dtype=I32, device="cuda") for m in ((n, width), n + 1, n, n, n, 1)]
    big = torch.zeros(1 << 26, device="cuda")
    seen = []
    for i in range(30):
        big.add_(1.0)                       # (work that takes a while, and then writes the lengths)
        cached.copy_((big[:n] * 16).to(I32))
        fresh.fill_(1)
        dvm.launch(code, [cached, fresh, free, *outs])
        dvm.launch(code, [outs[2], fresh, free, outs[0], *[torch.zeros_like(o) for o in outs[1:]]])   # reads the lengths just written
        seen.append((outs[2].clone(), outs[3].clone(), outs[5].clone()))
    ok()
    for i, (lengths, positions, taken) in enumerate(seen):
        assert (lengths == 16 * (i + 1) + 1).all() and (positions == 16 * (i + 1)).all() and int(taken) == n


def test_launches_wait_for_the_events_of_other_streams():
    """A kernel of its own stream right before, an event of another stream's long work between them."""
    n = 16
    code = dvm.encode_paging(n, 40, 16, n, 4096)
    cached, fresh, free = ints(np.zeros(n)), ints(np.ones(n)), torch.arange(4096, dtype=I32, device="cuda")
    outs = [torch.zeros(m, dtype=I32, device="cuda") for m in ((n, 40), n + 1, n, n, n, 1)]
    other = [torch.zeros_like(o) for o in outs]
    big = torch.zeros(1 << 26, device="cuda")
    mine, theirs = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    seen = []
    for i in range(20):
        with torch.cuda.stream(theirs):
            for _ in range(5):
                big.add_(0.2)
            cached.copy_((big[:n] + 0.5).to(I32) * 16)
            done = theirs.record_event()
        dvm.launch(code, [fresh, fresh, free, *other], mine)
        mine.wait_event(done)
        dvm.launch(code, [cached, fresh, free, *outs], mine)
        with torch.cuda.stream(mine):
            seen.append(outs[2].clone())
        theirs.wait_stream(mine)
    ok()
    assert all((x == 16 * (i + 1) + 1).all() for i, x in enumerate(seen))


@pytest.mark.parametrize("first", ["alone", "memset", "fork", "copy"])
def test_graphs_with_other_nodes(first):
    """A step (rotary, then attention of single tokens) captured behind nothing, a memset, a fork and a copy."""
    b = Batch([300, 40, 513], [1, 1, 1], 8, 2, 64, 16, seed=1)
    ang = angles(600, 64)
    pos, slots = ints([299, 39, 512]), ints([b.table[i, p // 16].item() * 16 + p % 16 for i, p in enumerate((299, 39, 512))])
    k, v = normal((3, 2, 64), BF16, 11), normal((3, 2, 64), BF16, 12)
    qr, out = torch.zeros_like(b.q), torch.zeros_like(b.q)
    rot = dvm.encode_rotary(q=b.q, k=k, v=v, angles=ang, q_out=qr, k_cache=b.k, v_cache=b.v)
    att = dvm.encode_attention(q=qr, k_cache=b.k, v_cache=b.v, table=b.table, out=out, scale=0.125, max_q=1)
    ws, lengths = torch.empty(dvm.tensor_extents(att)[-1], dtype=torch.uint8, device="cuda"), ints([300, 40, 513])
    s, side = torch.cuda.Stream(), torch.cuda.Stream()

    def step():
        dvm.launch(rot, [b.q, k, v, ang, pos, slots, qr, b.k, b.v], s)
        dvm.launch(att, [qr, b.k, b.v, b.table, b.starts, lengths, out, ws], s)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    want_q, want = qr.clone(), out.clone()
    kept = b.q.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        if first == "memset":
            qr.zero_()
        if first == "fork":
            side.wait_stream(s)
            with torch.cuda.stream(side):
                out.zero_()
            qr.zero_()
            s.wait_stream(side)
        if first == "copy":
            b.q.copy_(kept)
        step()
        step()
    for _ in range(3):
        g.replay()
        ok()
        assert torch.equal(qr, want_q) and torch.equal(out, want) and want.abs().sum() > 0


def test_eager_launches_on_two_streams_at_once():
    bs = [Batch([2000 + i, 900, 40], [1, 1, 1], 8, 2, 128, 16, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs, codes, ws, lengths = [], [], [], []
    for b in bs:
        outs.append([torch.zeros_like(b.q) for _ in range(20)])
        codes.append(b.code(outs[-1][0], scale=0.09, max_q=1))
        ws.append(torch.empty(dvm.tensor_extents(codes[-1])[-1], dtype=torch.uint8, device="cuda"))
        lengths.append(ints(b.lengths))
    torch.cuda.synchronize()
    for j in range(20):
        for b, s, o, c, w, n in zip(bs, streams, outs, codes, ws, lengths):
            dvm.launch(c, [b.q, b.k, b.v, b.table, b.starts, n, o[j], w], s)
    ok()
    for b, o, c in zip(bs, outs, codes):
        b.launch(c, last := torch.zeros_like(b.q))
        ok()
        assert all(torch.equal(x, last) for x in o) and last.abs().sum() > 0


def test_one_code_for_other_tensors_and_requests_that_share_pages():
    """A code holds a shape, not its tensors; two requests may read the same pages."""
    a = Batch([200, 200], [60, 60], 4, 2, 64, 16, seed=1)
    a.table[1, :8] = a.table[0, :8]
    a.check(max_q=60)
    b = Batch([200, 200], [60, 60], 4, 2, 64, 16, seed=2)
    out = torch.zeros_like(a.q)
    code = a.code(out, scale=0.125, max_q=60)
    for x in (b, a, b):
        x.launch(code, out)
        ok()
        want, mag, size, _, seen = orc.attention(f64(x.q), f64(x.k), f64(x.v), x.table.cpu().numpy(), x.starts.cpu().numpy(), x.lengths, 0.125, 0, 0)
        assert (np.abs(f64(out) - want) <= orc.attention_bound(want, mag, size, seen, 64, BF16, True)).all()


def test_debug_mode_checks_every_launch():
    """The variable is read once per process: the same operators in one of their own."""
    script = ("from tests.test_gpu_serving import Batch, check_rotary, paging_case, run_paging\n"
              "for fresh in (1, 30):\n"
              "    Batch([90, 70], [fresh] * 2, 4, 2, 64, 16).check(max_q=fresh)\n"
              "run_paging(*paging_case(33, 70, 40, 8, 1))\n"
              "check_rotary(5, 4, 2, 64, 64)\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", script], cwd=root, env=dict(os.environ, DVM_DEBUG="1"), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
