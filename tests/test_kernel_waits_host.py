"""Reads the kernel sources for two orders on which it depends that a kernel cannot wait for ever."""
import os
import re

import pytest

from paper_2105_09377_b200 import build

FILES = sorted(f for f in os.listdir(build.CSRC) if f.endswith((".cu", ".cuh")))


def _code(name):
    text = open(os.path.join(build.CSRC, name)).read()
    return re.sub(r"//[^\n]*", "", text)


def _kernels(text):
    """The text of every kernel, from its __global__ to the next one."""
    at = [m.start() for m in re.finditer(r"__global__", text)]
    return [text[a:b] for a, b in zip(at, at[1:] + [len(text)])]


@pytest.mark.parametrize("name", FILES)
def test_tensor_memory_is_allocated_before_the_next_kernel_may_start(name):
    """A kernel of the same stream that starts early allocates tensor memory too, and gives it back only after this one has
    ended: a block of this one that still waits for its own would wait for ever.  One thread's launch_dependents speaks
    for its block, so a barrier of the whole block has to lie between."""
    for kernel in _kernels(_code(name)):
        alloc = kernel.find("tcgen05.alloc")
        if alloc < 0:
            continue
        start = kernel.find("pdl_launch_dependents()", alloc)
        assert start > 0
        between = kernel[alloc:start]
        assert "__syncthreads()" in between or "cluster_sync_all()" in between, kernel[:200]


@pytest.mark.parametrize("name", FILES)
def test_roles_wait_for_one_another_with_a_limit(name):
    """A role that gives up after a bounded wait leaves for the end of the kernel.  A named barrier has no limit: the others
    would wait there for a warp that has left."""
    code = _code(name)
    assert not re.search(r"\b(bar|barrier)\.(cta\.)?sync\b|__barrier_sync|named_barrier", code)


@pytest.mark.parametrize("name", FILES)
def test_a_block_that_gave_up_lets_its_work_land(name):
    """Copies and matrix instructions in flight still write to the block's memory: it may neither leave nor give its tensor
    memory back right away.  Nor may it arm a barrier again whose copies never came."""
    for kernel in _kernels(_code(name)):
        if not re.search(r"abort_flag\s*=\s*reinterpret_cast", kernel) or "bounded_wait_selftest" in kernel[:200]:
            continue
        given_up = re.search(r"if \([^\n]*\*abort_flag\)", kernel)
        assert given_up and "global_timer()" in kernel[given_up.end():given_up.end() + 200], kernel[:200]
        dealloc = kernel.find("tcgen05.dealloc")
        assert dealloc < 0 or given_up.end() < dealloc
        if "attend_cache4(" in kernel[:120]:      # (the one kernel that fills its rings again after joining its warps)
            assert "if (__syncthreads_or(!ok)) break;" in kernel
