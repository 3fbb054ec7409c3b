"""Refusals, sizes and plans of the RMS norm, 8-bit matrices and the 8-bit linear layer that need no device."""
import glob
import os
import re

import numpy as np
import pytest

import ff_ref as R
from ff_ref import refused
from paper_2001_00138_b200 import binding as B, build

E_NULL, E_SHAPE, E_DTYPE = 1, 2, 9


def test_the_grid_of_eight_bits():
    assert len(R.GRID) == 127 and R.GRID[-1] == 448 and R.GRID[1] == 2.0 ** -9 and (np.diff(R.GRID) > 0).all()
    x = np.zeros((1, 200))
    x[0, 0], x[0, 1], x[0, 130] = 448.0, 17.0, 449.0       # 17: middle of 16 and 18, whose code is odd; 449 doubles the scale
    q = R.quantise8(x)
    assert q[0, 0] == 448 and q[0, 1] == 16 and q[0, 130] == 448


@pytest.mark.parametrize("kw", [dict(C=0), dict(C=65537), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(x_row=63), dict(r_row=-64),
                                dict(y_row=2 ** 31 + 1)])
def test_rms_refuses_sizes_and_strides(kw):
    refused(E_SHAPE, B.RmsNorm, **(dict(C=64) | kw))


def test_rms_refuses_types():
    for t in (-1, 3):
        refused(E_DTYPE, B.RmsNorm, 64, dtype=t)


def test_mx8_sizes():
    # row tiles of 128 rows; column tiles of 128 columns; 512 scale bytes per row tile and four column tiles
    assert B.mx8_bytes(0, 32) == 0
    assert B.mx8_bytes(1, 1) == B.mx8_bytes(128, 128) == 128 * 128 + 512
    assert B.mx8_bytes(129, 64) == 2 * (128 * 128 + 512)
    assert B.mx8_bytes(1, 129) == 2 * 128 * 128 + 512
    assert B.mx8_bytes(1, 513) == 5 * 128 * 128 + 2 * 512
    refused(E_SHAPE, B.mx8_bytes, -1, 32)
    refused(E_SHAPE, B.mx8_bytes, 1, 0)
    refused(E_SHAPE, B.mx8_bytes, 1, 2 ** 20 + 1)
    refused(E_SHAPE, B.mx8_bytes, 2 ** 31, 1)


@pytest.mark.parametrize("call", [B.mx8_quantize, B.mx8_dequantize])
def test_mx8_refusals(call):
    refused(E_DTYPE, call, 64, 64, 1, 32, dtype=7)
    refused(E_SHAPE, call, 64, 64, 1, 32, ld=31)
    refused(E_SHAPE, call, 64, 64, -1, 32)
    refused(E_SHAPE, B.mx8_quantize, 64, 72, 1, 32)           # the 8-bit buffer is not 16-byte aligned
    refused(E_SHAPE, B.mx8_dequantize, 72, 64, 1, 32)
    refused(E_SHAPE, B.mx8_quantize, 66, 64, 1, 32)           # a tensor that is not aligned to its elements
    refused(E_SHAPE, B.mx8_dequantize, 64, 66, 1, 32)
    refused(E_NULL, call, 0, 0, 1, 32)
    call(0, 0, 0, 32)                                         # no rows: nothing to do


@pytest.mark.parametrize("status, kw", [(E_SHAPE, dict(F=0)), (E_SHAPE, dict(K=0)), (E_SHAPE, dict(max_rows=-1)), (E_SHAPE, dict(ldw=63)),
                                        (E_SHAPE, dict(K=2 ** 21)), (E_SHAPE, dict(F=2 ** 21)), (E_DTYPE, dict(dtype=5)), (E_DTYPE, dict(act=9)),
                                        (E_NULL, dict(weights=0))])
def test_linear8_refusals(status, kw):
    refused(status, B.Linear8, **(dict(weights=64, F=32, K=64, max_rows=4) | kw))


def linear_sizes():
    rows = [1, 2, 8, 9, 16, 17, 48, 64, 65, 100, 128, 129, 300, 777, 3000, 20000]
    return [(f, k, m) for f in (1, 128, 130, 1000, 4096, 40000) for k in (1, 64, 65, 128, 129, 512, 1000, 4096, 25088, 1 << 20) for m in rows]


def test_ctas_of_the_8_bit_product_that_fit_an_sm_find_tensor_memory():
    """As for the 4-bit product: CTAs that fit an SM by their shared memory (228 KB, 1 KB of it kept per CTA) fit by their columns (512)."""
    clusters = 0
    for F, K, rows in linear_sizes():
        for mx in (False, True):
            p = B.linear8_plan(F, K, rows, from_8_bit_rows=mx)
            what = (F, K, rows, mx, p)
            columns = p["tensor_columns"]
            assert columns in (32, 64, 128, 256, 512), what
            used = p["tile_outputs"] + 12 * p["stages"] if p["persistent"] else p["tile_rows"] + 8 * p["stages"]
            assert used <= columns, what
            assert p["smem_bytes"] <= 226 * 1024, what
            if p["persistent"]:
                assert p["splits"] == 1, what
            else:
                assert (p["smem_bytes"] + 1024) * 512 >= columns * 228 * 1024, what
            clusters += p["splits"] > 1
    assert clusters > 100


def test_linear8_plan_refusals():
    for args in ((0, 32, 1), (32, 0, 1), (32, 32, 0), (32, 2 ** 21, 1), (2 ** 21, 32, 1), (2 ** 20, 1, 2 ** 31 - 1)):
        refused(E_SHAPE, B.linear8_plan, *args)


def allocating_kernels():
    """(file:name, body) of the kernels that take tensor memory through the shared helper."""
    found = []
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.cu"))):
        text = open(path).read()
        for m in re.finditer(r"__global__\b[^;{]*?\b(\w+_kernel)\s*\([^{;]*\)\s*\{", text):
            depth, at = 1, m.end()
            while depth:
                depth += {"{": 1, "}": -1}.get(text[at], 0)
                at += 1
            if "tmem_allocate" in text[m.end():at]:
                found.append((f"{os.path.basename(path)}:{m.group(1)}", text[m.end():at]))
    return found


@pytest.mark.parametrize("name, body", allocating_kernels(), ids=[n for n, _ in allocating_kernels()])
def test_dependents_start_after_the_allocation(name, body):
    """A dependent grid holds columns while it waits for this one: launch_dependents comes behind the barrier that publishes the allocation, which
    is made once and given back."""
    triggers = [m.start() for m in re.finditer(r"\bpdl_trigger\(\)", body)]
    barrier = body.index("__syncthreads()", body.index("tmem_allocate"))
    assert len(triggers) == 1 and triggers[0] > barrier
    assert len(re.findall(r"\btmem_allocate\w*\(", body)) == 1 and len(re.findall(r"\btmem_free\w*\(", body)) == 1


@pytest.mark.parametrize("status, kw", [(E_SHAPE, dict(F=0)), (E_SHAPE, dict(K=0)), (E_SHAPE, dict(max_rows=-1)), (E_SHAPE, dict(max_rows=2 ** 31)),
                                        (E_SHAPE, dict(x_row=63)), (E_SHAPE, dict(w_row=-64)), (E_SHAPE, dict(h_row=31)), (E_SHAPE, dict(h_row=2 ** 31 + 1)),
                                        (E_SHAPE, dict(K=2 ** 21)), (E_SHAPE, dict(F=2 ** 21)), (E_DTYPE, dict(dtype=B.F32)), (E_DTYPE, dict(dtype=5)),
                                        (E_DTYPE, dict(act=9))])
def test_gated_refusals(status, kw):
    refused(status, B.Gated, **(dict(F=32, K=64, max_rows=4) | kw))


def test_gated_plans():
    for F, K in ((1, 1), (64, 64), (130, 1000), (1333, 1000), (8192, 4096), (40000, 16384)):
        for rows in (1, 8, 100, 256, 300, 777, 5000, 100000):
            parts = [0, 0, 0]
            for product in range(3):
                p = B.gated_plan(F, K, rows, product)
                assert p["splits"] * p["blocks_per_split"] >= p["blocks"] > (p["splits"] - 1) * p["blocks_per_split"], p      # no range is empty
                tiles = p["row_tiles"] * p["column_tiles"]
                if p["few_rows"]:
                    assert product == 0 and p["grid"] == tiles * p["splits"] and p["splits"] <= 8
                    # the CTAs of a cluster wait for one another: where they fit an SM by shared memory they do by tensor memory
                    assert min(rows, 128) <= p["tensor_columns"] <= 128 and (p["smem_bytes"] + 1024) * 512 >= p["tensor_columns"] * 228 * 1024, p
                else:
                    parts[product] = tiles * p["splits"] if p["splits"] > 1 else 0
                    assert 2 <= p["grid"] <= 148 and p["grid"] % 2 == 0
                assert p["smem_bytes"] <= 226 * 1024
            assert parts[0] <= 148 and parts[1] + parts[2] <= 148           # units of partial sums that there is room for
    for args in ((0, 32, 1), (32, 0, 1), (32, 32, 0), (32, 2 ** 21, 1), (2 ** 21, 32, 1), (2 ** 20, 1, 2 ** 31 - 1)):
        refused(E_SHAPE, B.gated_plan, *args)
    refused(E_SHAPE, B.gated_plan, 32, 32, 1, 3)
