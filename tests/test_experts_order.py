"""What the sources of the operators of a layer of experts keep to so that no launch can hang or race: read from the text, since a
launch that breaks it may not be run."""
import os
import re

import pytest

from tests.test_experts_sources import SOURCES
from tests.test_kernel_resources import CSRC


def source(name):
    text = open(os.path.join(CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", text)


def calls(text, name):
    """Every call of `name`, with the text of its statement before it."""
    for m in re.finditer(r"\b%s\(" % name, text):
        start = max(text.rfind(c, 0, m.start()) for c in ";{}")
        yield text[start + 1: m.start()], m.start()


def inside_of(before, wrapper):
    """Whether the statement's beginning has an open bracket of `wrapper(`."""
    depth = 0
    for i in range(len(before) - 1, -1, -1):
        if before[i] == ")":
            depth += 1
        elif before[i] == "(":
            if depth == 0 and before[:i].rstrip().endswith(wrapper):
                return True
            depth -= depth > 0
    return False


@pytest.mark.parametrize("name", ["dvm_scaled_few.cu", "dvm_scaled_many.cu"])
def test_a_warp_gives_up_as_a_whole(name):
    """The lanes of a warp may see a limit run out, or the flag of those that gave up, at different turns: each wait of these kernels,
    whose warps go on to instructions of whole warps, is put to the vote."""
    text, seen = source(name), 0
    for wait in ("mbar_wait", "mbar_wait_flat", "mbar_poll"):
        for before, at in calls(text, wait):
            assert inside_of(before, "__all_sync"), text[at - 80: at + 60]
            seen += 1
    assert seen >= 3


def test_inside_of():
    assert inside_of("ok = __all_sync(ALL, a(b) && ", "__all_sync") and inside_of("__all_sync(ALL, (", "__all_sync")
    assert not inside_of("ok = __all_sync(ALL, a) && ", "__all_sync") and not inside_of("const bool ok = ", "__all_sync")
    assert SOURCES
