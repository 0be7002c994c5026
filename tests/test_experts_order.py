"""What the sources of the operators of a layer of experts keep to so that no launch can hang or race: read from the text, since a
launch that breaks it may not be run."""
import os
import re

import pytest

from tests.test_experts_sources import SOURCES
from tests.test_kernel_resources import CSRC, NVCC, _resources


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


# What a kernel may call before its wait for the launch before it: shared memory and barriers set up, descriptors of copies fetched,
# numbers formed, L2 asked for tiles.  Pointers among its arguments are not named there, but to ask whether there is one.
CALLS = {"if", "for", "sizeof", "smem_u32", "mbar_init", "tma_prefetch", "tma_ask_3d", "grid_ready", "range_of", "min", "max"}
ASM = {"mov.u32 %0, %%cluster_ctarank;", "fence.mbarrier_init.release.cluster;"}


def pointers(name):
    """The pointers among the kernels' arguments."""
    text = source("dvm_scaled.cuh" if "scaled" in name else name)
    fields = re.search(r"struct Args \{(.*?)\};", text, re.S).group(1)
    found = set()
    for line in fields.split(";"):
        if "*" in line:
            found |= set(re.findall(r"\*\s*(\w+)", line))
    return found


def kernels(name):
    text = source(name)
    heads = [m.start() for m in re.finditer(r"__global__", text)]
    for a, b in zip(heads, heads[1:] + [len(text)]):
        body = text[a:b]
        open_at = body.index("{", body.index("__grid_constant__ Args a"))
        depth, end = 0, open_at
        for end in range(open_at, len(body)):
            depth += {"{": 1, "}": -1}.get(body[end], 0)
            if depth == 0:
                break
        yield re.search(r"(dvm_\w+_kernel)\(", body).group(1), body[open_at: end + 1]


def early(body, pointer):
    """What a kernel does before its wait that it may not."""
    before = body[: body.index("grid_wait();")]
    found = [c for c in re.findall(r'asm(?: volatile)?\(\s*"([^"]*)"', before) if c not in ASM]
    plain = re.sub(r"\basm(?: volatile)?\([^;]*;[^;]*;", "", re.sub(r"if \(!a\.starts\)", "", before))
    plain = re.sub(r'"[^"]*"', "", plain)
    found += [c for c in re.findall(r"\b([A-Za-z_]\w*)(?:<[^<>()]*>)?\(", plain) if c not in CALLS]
    return found + [m for m in re.findall(r"\ba\.(\w+)", plain) if m in pointer]


@pytest.mark.parametrize("name", SOURCES)
def test_nothing_is_touched_before_the_wait(name):
    """Every kernel may start while the launch before it ends."""
    seen = 0
    for kernel, body in kernels(name):
        seen += 1
        assert body.count("grid_wait();") == 1 and body.index("grid_ready();") < body.index("grid_wait();"), kernel
        assert early(body, pointers(name)) == [], (kernel, early(body, pointers(name)))
        behind = body[body.index("grid_wait();"):]
        assert any(re.search(r"\ba\.%s\b" % p, behind) for p in pointers(name)), kernel
        asked = re.findall(r"tma_ask_3d\(([^;]*)\)", body[: body.index("grid_wait();")])
        assert all(a.startswith("&tm_w,") for a in asked) and (not asked or "if (!a.starts)" in body), kernel
    assert seen == source(name).count("__global__")


@pytest.mark.parametrize("name", SOURCES)
def test_what_comes_too_early_is_seen(name):
    """The same with the wait at the kernel's end, or behind a single access: the check sees it."""
    for kernel, body in kernels(name):
        without = body.replace("grid_wait();", "", 1)
        late = without[:-1] + "grid_wait();}"
        assert early(late, pointers(name)), kernel
        for line in ("const int x = a.%s[0];" % max(pointers(name)), "lay_out<1>(a, 1, 1, line, line);", "load_logits<2>(a, t, l);", "atomicAdd(a.status, 1u);",
                     "tma_load_3d(0, &tm_w, 0, 0, 0, 0);", 'asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(x) : "memory");',
                     "const float y = *a.%s;" % max(pointers(name)), "const T z = *(const T*)a.%s;" % min(pointers(name))):
            assert early(body.replace("grid_wait();", line + "\n  grid_wait();", 1), pointers(name)), (kernel, line)


@pytest.mark.skipif(not os.path.exists(NVCC), reason="nvcc not found")
def test_routing_spills_nothing():
    """Any number of experts: two CTAs of 512 threads per SM, and no register in memory."""
    res = {k: v for k, v in _resources("dvm_routing.cu").items() if "routing_kernelILi" in k}
    assert len(res) == 8 and any("ILi16E" in k for k in res)
    for name, (regs, _, stored, loaded) in res.items():
        assert regs <= 64 and stored == loaded == 0, (name, regs, stored, loaded)
