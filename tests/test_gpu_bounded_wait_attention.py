"""The attention kernels' bounded waits on real hardware, and the end of a CTA that gave up: copies still in flight are
awaited before it leaves its shared memory, whichever role's wait it was that ran out."""
import time

import pytest

import paper_2603_24239_b200 as dvm
from tests.test_gpu_serving import Batch

pytestmark = pytest.mark.gpu

DVM_ERR_DEVICE_TIMEOUT = -7


@pytest.mark.parametrize("which", [3, 4, 5])  # the waits of roles with their own registers, the short ones; the late copy
def test_wait_runs_out_and_reports(which):
    assert dvm.last_device_status() == 0
    t0 = time.perf_counter()
    dvm.selftest_bounded_wait(which)
    status = dvm.last_device_status()          # synchronises the stream
    dt = time.perf_counter() - t0
    assert status == DVM_ERR_DEVICE_TIMEOUT
    assert 1.0 < dt < 10.0, dt                 # the limit is 2 s
    assert dvm.last_device_status() == 0       # reading the status clears it
    for fresh in (1, 30):                      # the context is intact
        Batch([90, 70], [fresh] * 2, 4, 2, 64, 16).check(max_q=fresh)
