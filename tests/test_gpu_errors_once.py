"""A failed CUDA call is reported by the call it happened in, and by no later one."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

FAIL = '''
import torch
import dvm_workloads as wl
import paper_2603_24239_b200 as dvm
from tests.parity_util import check, gpu_run, oracle_run
from tests.test_gpu_serving import BF16, F32, Batch

def fail():
    """The host waits for a stream that is being captured: an error of that call, and the end of the capture."""
    s, g, before = torch.cuda.Stream(), torch.cuda.CUDAGraph(), torch.cuda.current_stream()
    try:
        with torch.cuda.graph(g, stream=s):
            try:
                dvm.last_device_status(s)
                raise SystemExit("the wait was allowed")
            except dvm.DvmError as e:
                assert e.status == -6 and dvm.lib.dvm_last_cuda_error() != 0
    except RuntimeError:
        pass
    torch.cuda.set_stream(before)
    torch.cuda.synchronize()
'''
ATTENTION = '''
b = Batch([90, 70], [{fresh}] * 2, 4, 2, 64, 16, dtype={dtype})
out = torch.zeros_like(b.q)
code, ws = b.code(out, scale=0.125, max_q={fresh}), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
dvm.launch(code, [b.q, b.k, b.v, b.table, b.starts, b.starts, out, ws])
torch.cuda.synchronize()
fail()
dvm.launch(code, [b.q, b.k, b.v, b.table, b.starts, b.starts, out, ws])
torch.cuda.synchronize()
'''
PROGRAM = '''
prog, ins = wl.program_c1(), wl.inputs_c1()
gpu_run(prog, ins)
fail()
outs, _ = gpu_run(prog, ins)
check(prog, outs, oracle_run(prog, ins))
'''


@pytest.mark.parametrize("name,then", [("plain", ATTENTION.format(fresh=1, dtype="F32")), ("plain", ATTENTION.format(fresh=30, dtype="F32")),
                                       ("single", ATTENTION.format(fresh=1, dtype="BF16")), ("prompt", ATTENTION.format(fresh=30, dtype="BF16")),
                                       ("program", PROGRAM)])
def test_the_next_launch_runs(name, then):
    """In a process of its own: a capture that ended this way leaves torch's allocator in a state that other tests need not have."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FAIL + then], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
