"""The work-queue slots go round among launches that have a queue: launches without one take none, or a serving loop would
bring a pending or captured stacked launch's counters to another one."""
import pytest
import torch

import dvm_workloads as wl
import paper_2603_24239_b200 as dvm
from tests.parity_util import gpu_run
from tests.test_gpu_serving import BF16, Batch, angles, check_rotary, normal, ok, paging_case, run_paging

pytestmark = pytest.mark.gpu


def stacked():
    dvm.set_elems_per_thread(16)
    try:
        codes, tls = [], []
        for j, (kind, r, c) in enumerate([("gelu_affine", 33, 300), ("layernorm", 17, 100)]):
            ins, params = wl.inputs_stack(kind, r, c, 40 + 4 * j)
            codes.append(dvm.encode(dvm.program_from_nodes(wl.stack_program(kind).nodes), [tuple(t.shape) for t in ins], params))
            tls.append([t.cuda() for t in ins] + [torch.empty((r, c), dtype=torch.float32, device="cuda")])
        dvm.launch_stacked(codes, tls)
    finally:
        dvm.set_elems_per_thread(0)


def test_only_launches_with_a_queue_take_a_slot():
    before = dvm.queue_slots_taken()
    run_paging(*paging_case(33, 70, 40, 8, 1))
    check_rotary(5, 4, 2, 64, 64)
    for fresh, kw in ((1, {}), (30, {}), (1, dict(dtype=torch.float32))):
        Batch([90, 70], [fresh] * 2, 4, 2, 64, 16, **kw).check(max_q=fresh)
    gpu_run(wl.program_mlp_gate(), [wl.randn((200, 256), torch.bfloat16, 3), wl.randn((256, 392), torch.bfloat16, 4, std=0.05),
                                    wl.randn((256, 392), torch.bfloat16, 5, std=0.05)])
    gpu_run(wl.program_c1(), wl.inputs_c1())
    ok()                                          # (reads the device's status)
    assert dvm.queue_slots_taken() == before
    stacked()
    ok()
    assert dvm.queue_slots_taken() == before + 1


def test_a_captured_stacked_launch_keeps_its_slot_to_itself():
    """A captured launch, 600 serving launches, and stacked launches beside its replays: each as if alone."""
    dvm.set_elems_per_thread(16)
    try:
        items = [("layernorm", 300 + i, 200) for i in range(6)]
        runs = []
        for seed in (0, 500):
            codes, tls = [], []
            for j, (kind, r, c) in enumerate(items):
                ins, params = wl.inputs_stack(kind, r, c, seed + 4 * j)
                codes.append(dvm.encode(dvm.program_from_nodes(wl.stack_program(kind).nodes), [tuple(t.shape) for t in ins], params))
                tls.append([t.cuda() for t in ins] + [torch.zeros((r, c), dtype=torch.float32, device="cuda")])
            dvm.launch_stacked(codes, tls)
            ok()
            runs.append((codes, tls, [t[-1].clone() for t in tls]))
    finally:
        dvm.set_elems_per_thread(0)
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        dvm.launch_stacked(runs[0][0], runs[0][1], side)
    q, k = normal((1, 4, 64), BF16, 1), normal((1, 2, 64), BF16, 2)
    ang, pos = angles(9, 64), torch.zeros(1, dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(q), torch.empty_like(k)
    code = dvm.encode_rotary(q=q, k=k, angles=ang, q_out=a, k_out=b)
    before = dvm.queue_slots_taken()
    for _ in range(600):
        dvm.launch(code, [q, k, ang, pos, a, b])
    assert dvm.queue_slots_taken() == before
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(side):
            g.replay()
        dvm.launch_stacked(runs[1][0], runs[1][1])
    ok()
    for _, tls, want in runs:
        assert all(torch.equal(t[-1], w) for t, w in zip(tls, want))
