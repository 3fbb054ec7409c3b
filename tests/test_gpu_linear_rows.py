"""The persistent kernel of the 4-bit product (many rows) in each of its forms: 128 and 256 outputs per tile, an odd last tile of weights, 32- and
64-byte pieces, column tiles beyond the ring, every activation, and rows of y that are aligned to 16, 4 and 2 bytes.

Rows and weights are values that 4 bits hold exactly, with a power of two per block, so the references need no quantisation; the fp32 sums are
held to the bound of test_gpu_mx4 ((K / 64 + 10) roundings of the sum of magnitudes, then the output's own).
"""
import pytest

import ops_ref as R

pytestmark = pytest.mark.gpu

FORMS = {  # rows, K, F, and what patdnn_linear_plan says
    "256 outputs, odd last tile, 64-byte pieces": (9500, 300, 513, dict(tile_outputs=256, piece_bytes=64, column_tiles=2)),
    "256 outputs, odd last tile, 32-byte pieces, ring wraps": (9500, 1100, 513, dict(tile_outputs=256, piece_bytes=32, column_tiles=5, stages=4)),
    "256 outputs, 64 columns": (19000, 64, 200, dict(tile_outputs=256, piece_bytes=64, column_tiles=1)),
    "256 outputs, 128 columns, odd last step": (19000, 90, 129, dict(tile_outputs=256, piece_bytes=64, column_tiles=1)),
    "256 outputs, several per CTA": (40000, 200, 600, dict(tile_outputs=256, piece_bytes=64, column_tiles=1)),
    "256 outputs, full tiles": (10000, 2048, 768, dict(tile_outputs=256, piece_bytes=32, column_tiles=8)),
    "128 outputs, 32-byte pieces, ring wraps": (20000, 2000, 100, dict(tile_outputs=128, piece_bytes=32, column_tiles=8, stages=6)),
    "128 outputs, odd last tile, 32-byte pieces": (3000, 1100, 1100, dict(tile_outputs=128, piece_bytes=32)),
    "128 outputs, 64-byte pieces": (20001, 700, 7, dict(tile_outputs=128, piece_bytes=64, column_tiles=3)),
}
ACTS = ["none", "relu", "silu"]


def held(rows, cols, g):
    """Values that blocks of 32 hold exactly: the eight magnitudes, both signs, times a power of two per block."""
    import torch
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda")
    v = grid[torch.randint(0, 8, (rows, cols), generator=g, device="cuda")] * (torch.randint(0, 2, (rows, cols), generator=g, device="cuda") * 2 - 1)
    e = torch.randint(-3, 4, (rows, -(-cols // 32)), generator=g, device="cuda").repeat_interleave(32, 1)[:, :cols]
    return torch.ldexp(v, e)


@pytest.mark.parametrize("aligned", [16, 4, 2])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", FORMS)
def test_many_rows(form, dtype, aligned):
    import torch
    from paper_2001_00138_b200 import binding as B
    rows, K, F, plan = FORMS[form]
    tt, dt = {"f32": (torch.float32, B.F32), "f16": (torch.float16, B.F16), "bf16": (torch.bfloat16, B.BF16)}[dtype]
    st = torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device="cuda").manual_seed(K + F)
    x, w, b = held(rows, K, g), held(F, K, g) / 8, torch.randn(F, generator=g, device="cuda")
    # elements between rows of y, and before its first: 16-byte rows, rows of whole pairs, odd ones
    ldy, first = {16: (-(-F // 8) * 8 + 8, 8), 4: (-(-F // 8) * 8 + 2, 2), 2: (-(-F // 8) * 8 + 1, 1)}[aligned]
    for n, act in enumerate(ACTS):
        mx = (n + aligned) % 2 == 0
        got = B.linear_plan(F, K, rows, from_4_bit_rows=mx)
        assert got["persistent"] == 1 and {k: got[k] for k in plan} == plan, got
        lin = B.Linear(w.to(tt), F, K, max_rows=0 if mx else rows, dtype=dt, bias=b if n else None, act=[B.ACT_NONE, B.ACT_RELU, B.ACT_SILU][n], stream=st)
        flat = torch.full((first + rows * ldy + 64,), float("nan"), dtype=tt, device="cuda")
        y = torch.as_strided(flat, (rows, F), (ldy, 1), first)
        if mx:
            buf = torch.full((B.mx4_bytes(rows, K),), 255, dtype=torch.uint8, device="cuda")
            B.mx4_quantize(x.to(tt), buf, rows, K, dtype=dt, stream=st)
            lin.run_mx4(buf, y, rows, ldy=ldy, stream=st)
        else:
            lin.run(x.to(tt), y, rows, ldy=ldy, stream=st)
        lin.check()
        bias = b.double() if n else torch.zeros(F, dtype=torch.float64, device="cuda")
        z = x.double() @ w.double().t() + bias
        ref = z if act == "none" else z.clamp_min(0) if act == "relu" else z / (1 + torch.exp(-z))
        size = x.double().abs() @ w.double().abs().t() + bias.abs()
        bound = 1.1 * (K / 64 + 10) * 2.0 ** -23 * size + R.UNIT[dtype] * ref.abs() * 1.01 + R.TINY[dtype]
        off = (y.double() - ref).abs()
        bad = ~(off <= bound)
        assert not bad.any(), (act, int(bad.sum()), bad.nonzero()[:4].tolist(), off[bad][:4].tolist(), bound[bad][:4].tolist())
        inside = torch.zeros_like(flat, dtype=torch.bool)
        torch.as_strided(inside, y.shape, y.stride(), first).fill_(True)
        assert torch.isnan(flat[~inside]).all(), act


def test_a_row_that_is_not_finite_spoils_no_other():
    import torch
    from paper_2001_00138_b200 import binding as B
    rows, K, F = 9500, 600, 513
    assert B.linear_plan(F, K, rows)["persistent"] == 1
    st = torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w = torch.randn(rows, K, generator=g, device="cuda"), torch.randn(F, K, generator=g, device="cuda")
    lin = B.Linear(w, F, K, max_rows=rows, stream=st)
    y0, y1 = torch.empty(rows, F, device="cuda"), torch.empty(rows, F, device="cuda")
    lin.run(x, y0, rows, stream=st)
    hit = [0, 127, 128, 5000, 9499]
    for i, r in enumerate(hit):
        x[r, 100 * i + 33] = [float("inf"), float("nan"), float("-inf")][i % 3]
    lin.run(x, y1, rows, stream=st)
    lin.check()
    others = torch.ones(rows, dtype=torch.bool, device="cuda")
    others[hit] = False
    assert torch.isnan(y1[hit]).all() and torch.isfinite(y0).all()
    assert torch.equal(y1[others], y0[others])
