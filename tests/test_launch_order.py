"""Kernels that take tensor memory let their successor start only once every block has it.

A successor may take tensor memory before it waits for its predecessor.  If a block let it start with its own allocation still
to come, the successor could take the columns on that SM and wait for the block, and the block for the columns: neither would
end.  So the signal has to stand behind a barrier of the whole block that stands behind the allocation.  That is an order of
statements, and is read in the sources: a run would only hang, and only where the two happen to meet on an SM.

(ffn_matmul_kernel, which signals through a function of its own, is always followed by a kernel of the same call that takes no
tensor memory.)"""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_21198_b200", "csrc")
ALLOCATES = re.compile(r"\btmem_alloc\(|tcgen05\.alloc\b")
LETS_START = re.compile(r"\bafter_predecessor\(\)|\blet_successor\(\)|griddepcontrol\.launch_dependents")


def kernels(text):
    """(name, body) of every __global__ function, comments left out."""
    text = re.sub(r"//[^\n]*", "", text)
    for start in re.finditer(r"__global__", text):
        at, depth = text.index("{", start.end()), 0
        name = re.search(r"(\w+)\s*\((?:[^()]|\([^()]*\))*\)\s*$", text[start.end():at]).group(1)
        for end in range(at, len(text)):
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            if depth == 0:
                break
        yield name, text[at:end]


def found():
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        for name, body in kernels(open(path).read()):
            if ALLOCATES.search(body) and LETS_START.search(body):
                yield pytest.param(body, id=name)


def test_the_kernels_are_found():
    assert {p.id for p in found()} >= {"router_kernel", "resident_ffn_kernel", "grouped_few_kernel", "grouped_wide_kernel"}


@pytest.mark.parametrize("body", list(found()))
def test_successors_start_behind_the_allocation(body):
    allocated = ALLOCATES.search(body).end()
    barrier = body.find("__syncthreads()", allocated)
    first = LETS_START.search(body).start()
    assert allocated < barrier < first, "lets its successor start before all of the block have the tensor memory"
