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


def linear_sizes():
    rows = [1, 2, 8, 9, 16, 17, 48, 64, 65, 100, 128, 129, 300, 777, 3000, 20000]
    return [(f, k, m) for f in (1, 128, 130, 1000, 4096, 40000) for k in (1, 64, 65, 128, 129, 512, 1000, 4096, 25088, 1 << 20) for m in rows]


def test_ctas_that_fit_an_sm_find_tensor_memory():
    """The CTAs of a cluster wait for one another while they hold columns: CTAs of the product that fit an SM by their shared memory (228 KB,
    1 KB of it kept per CTA) fit by their columns (512), whatever other such CTA is there."""
    from paper_2001_00138_b200 import binding as B
    clusters = 0
    for F, K, rows in linear_sizes():
        for mx in (False, True):
            p = B.linear_plan(F, K, rows, from_4_bit_rows=mx)
            what = (F, K, rows, mx, p)
            columns = p["tensor_columns"]
            assert columns in (32, 64, 128, 256, 512), what
            wide = p["tile_outputs"] // 128
            used = p["tile_outputs"] + (8 + 8 * wide) * p["stages"] if p["persistent"] else p["tile_rows"] + 16 * p["stages"]
            assert used <= columns, what
            assert p["smem_bytes"] <= 226 * 1024, what
            if p["persistent"]:
                assert p["splits"] == 1, what              # waits for nothing but earlier grids
            else:
                assert (p["smem_bytes"] + 1024) * 512 >= columns * 228 * 1024, what
            clusters += p["splits"] > 1
    assert clusters > 100


def test_linear_plan_refusals():
    from paper_2001_00138_b200 import binding as B
    for args in ((0, 32, 1), (32, 0, 1), (32, 32, 0), (32, 2 ** 21, 1), (2 ** 21, 32, 1), (2 ** 20, 1, 2 ** 31 - 1)):
        with pytest.raises(B.PatdnnError) as e:
            B.linear_plan(*args)
        assert e.value.status == 2
