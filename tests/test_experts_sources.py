"""What the compiler made of the kernels of a layer of experts (`-Xptxas -v`), and what their sources keep to that no launch can
show without risk."""
import os
import re

import pytest

from tests.test_kernel_resources import CSRC, NVCC, _resources

SOURCES = ["dvm_combine.cu", "dvm_quantize.cu", "dvm_routing.cu", "dvm_scaled_few.cu", "dvm_scaled_many.cu"]


def bodies(name):
    text = open(os.path.join(CSRC, name)).read()
    starts = [m.start() for m in re.finditer(r"__global__", text)] + [len(text)]
    return [text[a:b] for a, b in zip(starts, starts[1:])]


@pytest.mark.skipif(not os.path.exists(NVCC), reason="nvcc not found")
@pytest.mark.parametrize("source,kernel,count,least,most,spilled", [
    ("dvm_routing.cu", "routing_kernelILi2E", 2, 1, 64, 0),     # two CTAs of 512 threads per SM
    ("dvm_routing.cu", "routing_kernelILi4E", 2, 1, 64, 0),
    ("dvm_routing.cu", "routing_kernelILi8E", 2, 1, 64, 64),    # (off the keys' sort: what a warp keeps of the chunk)
    ("dvm_routing.cu", "routing_joint_kernel", 8, 1, 128, 0),   # one
    ("dvm_routing.cu", "routing_plan_kernel", 1, 1, 128, 0),
    ("dvm_quantize.cu", "quantize_kernel", 8, 1, 64, 0),        # four CTAs of 256 threads per SM
    ("dvm_quantize.cu", "quantize_block_kernel", 4, 1, 128, 0),
    ("dvm_scaled_few.cu", "scaled_few_kernel", 2, 1, 168, 0),
    ("dvm_scaled_few.cu", "scaled_join_kernel", 2, 1, 64, 0),
    ("dvm_scaled_many.cu", "scaled_many_kernel", 2, 168, 168, 256),   # 384 threads: what setmaxnreg deals out by role is counted from this
    ("dvm_combine.cu", "combine_kernel", 4, 1, 128, 0),
])
def test_registers_and_spills(source, kernel, count, least, most, spilled):
    res = {k: v for k, v in _resources(source).items() if kernel in k}
    assert len(res) == count, list(res)
    for name, (regs, stack, st, ld) in res.items():
        assert least <= regs <= most, (name, regs)
        assert st <= spilled and ld <= spilled, (name, stack, st, ld)


@pytest.mark.parametrize("name", SOURCES)
def test_every_kernel_waits_for_the_launch_before(name):
    """Every kernel may start while the one before it ends: it touches memory, and asks for tensor memory, behind its wait only."""
    kernels = bodies(name)
    assert kernels
    for body in kernels:
        wait = body.index("grid_wait();")
        for word in (r"tcgen05\.alloc", r"cp\.async", r"ld_global|__ldg|__ldcs"):
            assert all(wait < m.start() for m in re.finditer(word, body)), word


def test_what_the_many_rows_kernel_deals_out():
    text = open(os.path.join(CSRC, "dvm_scaled_many.cu")).read()
    of = lambda name: int(re.search(r"\b%s = (\d+)" % name, text).group(1))  # noqa: E731
    assert of("MANY_THREADS") == 384 and 256 * of("SUM_REGS") + 128 * of("OTHER_REGS") <= 384 * 168


@pytest.mark.parametrize("name", SOURCES + ["dvm_scaled.cu", "dvm_scaled.cuh", "dvm_experts_launch.h"])
def test_no_wait_of_its_own(name):
    """Waits for barriers are those of the shared header, which count their turns."""
    text = open(os.path.join(CSRC, name)).read()
    assert not re.search(r"mbarrier\.(try|test)_wait|multicast|__trap|\bassert\(", text)
