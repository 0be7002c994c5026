"""What the sources of the serving kernels keep to and no launch can show without risk."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2603_24239_b200", "csrc")
EARLY = [f for f in sorted(os.listdir(CSRC)) if f.endswith(".cu") and "dvm_launch_early(" in open(os.path.join(CSRC, f)).read()]


def kernels(name):
    text = open(os.path.join(CSRC, name)).read()
    starts = [m.start() for m in re.finditer(r"__global__", text)] + [len(text)]
    return [text[a:b] for a, b in zip(starts, starts[1:]) if "grid_wait();" in text[a:b]]


def test_early_kernels_are_found():
    assert EARLY == ["dvm_attention_prompt.cu", "dvm_attention_single.cu", "dvm_paging.cu", "dvm_rotary.cu"]
    assert [len(kernels(f)) for f in EARLY] == [1, 2, 1, 1]


@pytest.mark.parametrize("name", EARLY)
def test_tensor_memory_is_asked_for_behind_the_wait(name):
    """A kernel that starts while the one before it ends must not hold tensor memory that the other is about to ask for."""
    for body in kernels(name):
        for m in re.finditer(r"tcgen05\.alloc", body):
            assert body.index("grid_wait();") < m.start()
