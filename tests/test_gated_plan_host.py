"""How the gated block reads weights whose rows are not whole 16-byte units apart, without a device."""
import pytest

from ff_ref import refused
from paper_2001_00138_b200 import binding as B

E_SHAPE = 2


def phases(w_row):
    """Every how manieth row begins at the same place of a 16-byte unit."""
    return 1 if w_row % 8 == 0 else 2 if w_row % 4 == 0 else 4 if w_row % 2 == 0 else 8


def test_plans_of_weights_that_are_read_as_they_lie():
    """Few rows: tiles of 64 rows of ONE phase, seven columns more than K to shift by; memory limits as for aligned weights."""
    seen = set()
    for F, K in ((1, 1), (8, 100), (64, 64), (130, 1001), (1333, 1003), (4222, 6899), (8192, 4098), (40000, 16383)):
        for w_row in (K, K + 1, K + 2, K + 4, K + 8):
            for rows in (1, 8, 60, 100, 128, 129, 777):
                p, plain = B.gated_plan(F, K, rows, 0, w_row), B.gated_plan(F, K, rows, 0)
                n = phases(w_row)
                if n == 1 or rows > 128 or n > F or K + 8 > n * w_row or n * rows > F:
                    assert p == plain
                    continue
                seen.add((n, p["splits"]))
                assert p["few_rows"] == 1 and p["row_tiles"] == 1 and p["column_tiles"] == n * -(-(-(-F // n)) // 64) and p["blocks"] == -(-(K + 7) // 64)
                assert p["grid"] == p["column_tiles"] * p["splits"] and p["splits"] in (1, 2, 4, 8)
                assert p["splits"] * p["blocks_per_split"] >= p["blocks"] and 1 <= p["stages"] <= max(1, p["blocks_per_split"])
                assert rows <= p["tensor_columns"] <= 128 and p["smem_bytes"] <= 226 * 1024
                # the CTAs of a cluster wait for one another: where they fit an SM by shared memory they do by tensor memory
                assert (p["smem_bytes"] + 1024) * 512 >= p["tensor_columns"] * 228 * 1024, p
            for product in (1, 2):
                assert B.gated_plan(F, K, 40, product, w_row) == B.gated_plan(F, K, 40, product)
    assert {n for n, _ in seen} == {2, 4, 8} and {s for _, s in seen} >= {1, 2, 4}, seen


def test_refusals():
    for w_row in (31, -32, 2 ** 31 + 1):
        refused(E_SHAPE, B.gated_plan, 64, 32, 1, 0, w_row)
    refused(E_SHAPE, B.gated_plan, 64, 32, 1, 3, 33)
