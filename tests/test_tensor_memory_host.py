"""Tensor memory is allocated with a blocking instruction, the one wait of the tensor-core kernels that has no bound of its own.  These checks
show, without a device, that it always ends."""
import glob
import os
import re

import pytest

from paper_2001_00138_b200 import build

CSRC = build.CSRC


def kernels():
    """(file:name, body) of every kernel that allocates tensor memory."""
    found = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        text = open(path).read()
        for m in re.finditer(r"__global__\b[^;{]*?\b(\w+_kernel)\s*\([^{;]*\)\s*\{", text):
            depth, at = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(text[at], 0)
                at += 1
            body = text[m.end():at]
            if "tcgen05.alloc" in body:
                found.append((f"{os.path.basename(path)}:{m.group(1)}", body))
    return found


def test_the_kernels_are_found():
    assert len(kernels()) == 6


@pytest.mark.parametrize("name, body", kernels(), ids=[n for n, _ in kernels()])
def test_dependents_start_after_the_allocation(name, body):
    """A dependent grid holds its own columns while it waits for this one, so none of its CTAs may arrive before every CTA here holds its
    columns: launch_dependents (where a kernel gives it at all) comes behind the barrier that publishes the allocation."""
    triggers = [m.start() for m in re.finditer(r"\bpdl_trigger\(\)", body)]
    assert len(triggers) <= 1
    alloc = body.index("tcgen05.alloc")
    barrier = body.index("__syncthreads()", alloc)
    assert all(t > barrier for t in triggers)
    assert "tcgen05.alloc" not in body[alloc + 1:]
