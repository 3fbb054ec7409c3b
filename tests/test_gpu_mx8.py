"""8-bit matrices and the linear layer on them against 64-bit statements.

Quantised values are whole multiples of a power of two and have to be equal; the products' bound is that of ff_ref.product_bound, fixed
before the first run.
"""
import numpy as np
import pytest

import ff_ref as R
from ff_ref import held8, mx8_buffer, product_bound, refused, spaced, stream, types, untouched

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "silu"]
E_DEVICE_TIMEOUT = 8


def act_of(name):
    from paper_2001_00138_b200 import binding as B
    return [B.ACT_NONE, B.ACT_RELU, B.ACT_SILU][ACTS.index(name)]


SIZES = [(20001, 60), (5003, 127), (3001, 250), (30000, 8), (1, 1), (1, 31), (3, 32), (2, 33), (8, 63), (33, 64), (128, 65), (129, 128), (31, 129), (97, 200), (5, 256), (7, 511), (256, 513), (130, 2049), (40, 4096)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("slack, offset", [(0, 0), (8, 0), (2, 2), (3, 1), (5, 7), (1, 6)])
def test_quantise_and_back(rows, cols, dtype, slack, offset):
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = types(dtype)
    g = torch.Generator().manual_seed(rows * 1000 + cols)
    x = (torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-6, 6, (rows, 1), generator=g).float())).to(tt)
    _, v = spaced(x, slack, offset)
    mx = mx8_buffer(rows, cols)
    B.mx8_quantize(v, mx, rows, cols, dtype=dt, ld=cols + slack, stream=stream())
    flat, out = spaced(torch.zeros(rows, cols, dtype=tt), slack, offset)
    B.mx8_dequantize(mx, out, rows, cols, dtype=dt, ld=cols + slack, stream=stream())
    torch.cuda.synchronize()
    want = torch.from_numpy(R.quantise8(x.double().numpy())).to(tt)      # (exact but for small halves, which round once)
    assert torch.equal(out.cpu(), want)
    assert untouched(flat, out)


def round_trip(x):
    import torch
    from paper_2001_00138_b200 import binding as B
    rows, cols = x.shape
    mx, out = mx8_buffer(rows, cols), torch.empty(rows, cols, device="cuda")
    B.mx8_quantize(x.cuda(), mx, rows, cols, stream=stream())
    B.mx8_dequantize(mx, out, rows, cols, stream=stream())
    torch.cuda.synchronize()
    return out.cpu().double().numpy()


def test_ties_signs_and_extreme_scales():
    import torch
    # every value of the grid, every middle of two neighbours, and their surroundings, under block maxima around 448 and 256
    points = np.concatenate([R.GRID, R.MIDDLE, R.MIDDLE * (1 + 2.0 ** -20), R.MIDDLE * (1 - 2.0 ** -20)])
    points = np.concatenate([points, -points])
    for top in (448.0, np.nextafter(np.float32(448), np.float32(1000)), 447.0, 256.0, 255.99, 300.0):
        inside = points[np.abs(points) <= top]
        inside = np.concatenate([inside, np.zeros(-len(inside) % 127)]).reshape(-1, 127)
        x = np.concatenate([np.full((len(inside), 1), top), inside], axis=1)
        for e in (0, -149 - 8, -140, -135, -128, -127, -126, -125, -119, -118, -60, 60, 110, 118):
            y = torch.from_numpy(np.ldexp(x, e)).float()
            assert torch.isfinite(y).all()
            assert np.array_equal(round_trip(y), R.quantise8(y.double().numpy())), (top, e)
    assert not round_trip(torch.zeros(4, 300)).any()


def test_the_largest_floats():
    """Magnitudes that round up to 2^128 read back as infinities."""
    import torch
    x = torch.zeros(2, 128)
    x[0, 0], x[0, 1] = 3.4e38, 1.0e38
    x[1, 0] = 3.2e38
    got = round_trip(x)
    assert np.isinf(got[0, 0]) and got[0, 1] == R.quantise8(x.double().numpy())[0, 1] and got[1, 0] == R.quantise8(x.double().numpy())[1, 0]


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_not_finite_blocks(bad):
    import torch
    x = torch.randn(40, 300, generator=torch.Generator().manual_seed(1))
    x[7, 140] = bad
    x[39, 299] = bad
    got, ref = round_trip(x), R.quantise8(x.double().numpy())
    assert np.isnan(ref[7, 128:256]).all() and np.isnan(ref[39, 256:]).all() and np.isnan(ref).sum() == 128 + 44
    assert np.array_equal(got, ref, equal_nan=True)


def linear_case(M, K, F, dtype, act, *, slack=0, seed=0, bias=True, mx=False):
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = types(dtype)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g).to(tt)
    w = (torch.randn(F, K, generator=g) / K ** 0.5).to(tt)
    b = torch.randn(F, generator=g)
    _, xv = spaced(x, slack)
    _, wv = spaced(w, slack)
    flat, y = spaced(torch.zeros(M, F, dtype=tt), slack)
    lin = B.Linear8(wv, F, K, max_rows=M, dtype=dt, bias=b.cuda() if bias else None, act=act_of(act), ldw=K + slack, stream=stream())
    if mx:
        buf = mx8_buffer(M, K)
        B.mx8_quantize(xv, buf, M, K, dtype=dt, ld=K + slack, stream=stream())
        lin.run_mx8(buf, y, M, ldy=F + slack, stream=stream())
    else:
        lin.run(xv, y, M, ldx=K + slack, ldy=F + slack, stream=stream())
    lin.check()
    xq, wq = R.quantise8(x.double().numpy()), R.quantise8(w.double().numpy())
    z = xq @ wq.T + (b.double().numpy() if bias else 0)
    ref = R.act(z, act)
    size = np.abs(xq) @ np.abs(wq).T + np.abs(b.double().numpy())
    R.within(y.double().cpu().numpy(), ref, product_bound(K, size, ref, dtype), f"{M} x {K} x {F} {dtype} {act}")
    assert untouched(flat, y)
    lin.free()


@pytest.mark.parametrize("M, K, F", [
    (1, 1, 1), (1, 32, 128), (1, 4096, 130), (2, 64, 64), (3, 100, 7), (4, 4100, 1000), (8, 2500, 300), (9, 700, 512), (15, 129, 257), (16, 256, 128), (17, 1000, 200),
    (32, 8192, 256), (33, 512, 384), (64, 96, 1000), (100, 3000, 100), (128, 640, 640), (129, 64, 128), (255, 300, 300), (256, 1024, 256), (257, 128, 129), (500, 65, 500),
    (1000, 1000, 1000), (5000, 64, 256), (3000, 520, 1100), (20000, 40, 24)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_linear(M, K, F, dtype):
    linear_case(M, K, F, dtype, ACTS[(M + K + F) % 3], seed=M + K, bias=(M + F) % 4 != 0)


@pytest.mark.parametrize("M, K, F", [(1, 300, 130), (40, 300, 130), (300, 300, 300), (2000, 128, 512)])
@pytest.mark.parametrize("dtype, slack", [("f32", 8), ("f32", 1), ("f16", 8), ("bf16", 3)])
def test_linear_strides_and_8_bit_rows(M, K, F, dtype, slack):
    linear_case(M, K, F, dtype, "relu", slack=slack, seed=5)
    linear_case(M, K, F, dtype, "silu", slack=slack, seed=6, mx=True)


FORMS = {  # rows, K, F, 8-bit rows, and what patdnn_linear8_plan says
    "quantises its rows, cluster of four": (3, 1100, 100, False, dict(quantises=1, splits=4, column_tiles=9)),
    "quantises its rows, one tile": (8, 60, 30000, False, dict(quantises=1, splits=1)),
    "a cluster of eight": (40, 8192, 256, True, dict(persistent=0, splits=8)),
    "a cluster of eight, many rows": (128, 16384, 300, False, dict(persistent=0, splits=8, tile_rows=128)),
    "a cluster of two, uneven": (200, 2300, 4000, True, dict(persistent=0, splits=2, column_tiles=18)),
    "a cluster of four, uneven": (200, 2300, 400, True, dict(persistent=0, splits=4, column_tiles=18)),
    "no cluster, ring wraps": (300, 1500, 700, True, dict(persistent=0, splits=1, column_tiles=12)),
    "256 outputs, odd last tile": (9500, 300, 513, True, dict(persistent=1, tile_outputs=256, column_tiles=3)),
    "256 outputs, ring wraps": (9500, 1100, 513, False, dict(persistent=1, tile_outputs=256, column_tiles=9)),
    "256 outputs, one column tile": (40000, 90, 600, True, dict(persistent=1, tile_outputs=256, column_tiles=1)),
    "256 outputs, full tiles": (10000, 1024, 768, True, dict(persistent=1, tile_outputs=256, column_tiles=8)),
    "256 outputs, few of them": (20000, 2000, 100, True, dict(persistent=1, tile_outputs=256, column_tiles=16)),
    "256 outputs, fewer tiles than pairs": (3000, 1100, 1100, True, dict(persistent=1, tile_outputs=256, grid=120)),
    "no cluster, several tiles of rows": (1000, 300, 300, True, dict(persistent=0, splits=1, tile_rows=128)),
}


@pytest.mark.parametrize("aligned", [16, 4, 2])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("form", FORMS)
def test_every_form(form, dtype, aligned):
    """Values that 8 bits hold exactly, so that the reference is a plain product; rows of y aligned to 16, 4 and 2 bytes."""
    import torch
    from paper_2001_00138_b200 import binding as B
    rows, K, F, mx, plan = FORMS[form]
    tt, dt = types(dtype)
    g = torch.Generator(device="cuda").manual_seed(K + F)
    x, w, b = held8(rows, K, g), held8(F, K, g) / 32, torch.randn(F, generator=g, device="cuda")
    ldy, first = {16: (-(-F // 8) * 8 + 8, 8), 4: (-(-F // 8) * 8 + 2, 2), 2: (-(-F // 8) * 8 + 1, 1)}[aligned]
    got = B.linear8_plan(F, K, rows, from_8_bit_rows=mx)
    assert {k: got[k] for k in plan} == plan, got
    for n, act in enumerate(ACTS):
        lin = B.Linear8(w.to(tt), F, K, max_rows=0 if mx else rows, dtype=dt, bias=b if n else None, act=act_of(act), stream=stream())
        flat = torch.full((first + rows * ldy + 64,), float("nan"), dtype=tt, device="cuda")
        y = torch.as_strided(flat, (rows, F), (ldy, 1), first)
        if mx:
            buf = mx8_buffer(rows, K)
            B.mx8_quantize(x.to(tt), buf, rows, K, dtype=dt, stream=stream())
            lin.run_mx8(buf, y, rows, ldy=ldy, stream=stream())
        else:
            lin.run(x.to(tt), y, rows, ldy=ldy, stream=stream())
        lin.check()
        bias = b.double() if n else torch.zeros(F, dtype=torch.float64, device="cuda")
        z = x.double() @ w.double().t() + bias
        ref = z if act == "none" else z.clamp_min(0) if act == "relu" else z / (1 + torch.exp(-z))
        bound = product_bound(K, x.double().abs() @ w.double().abs().t() + bias.abs(), ref, dtype)
        off = (y.double() - ref).abs()
        bad = ~(off <= bound)
        assert not bad.any(), (act, int(bad.sum()), bad.nonzero()[:4].tolist(), off[bad][:4].tolist(), bound[bad][:4].tolist())
        assert untouched(flat, y), act


@pytest.mark.parametrize("M, K, F", [(1, 600, 200), (5, 600, 200), (40, 600, 200), (300, 600, 200), (9500, 600, 513)])
def test_a_row_that_is_not_finite_spoils_no_other(M, K, F):
    import torch
    from paper_2001_00138_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(F, K, generator=g, device="cuda")
    lin = B.Linear8(w, F, K, max_rows=M, stream=stream())
    y0, y1 = torch.empty(M, F, device="cuda"), torch.empty(M, F, device="cuda")
    lin.run(x, y0, M, stream=stream())
    hit = sorted({0, M // 2, M - 1})
    for i, r in enumerate(hit):
        x[r, 200 * i + 33] = [float("inf"), float("nan"), float("-inf")][i]
    lin.run(x, y1, M, stream=stream())
    lin.check()
    others = torch.ones(M, dtype=torch.bool, device="cuda")
    others[hit] = False
    assert torch.isnan(y1[hit]).all() and torch.isfinite(y0).all()
    assert torch.equal(y1[others], y0[others])


def test_fewer_rows_than_the_handle_was_made_for_and_refusals():
    import torch
    from paper_2001_00138_b200 import binding as B
    K, F = 384, 96
    g = torch.Generator(device="cuda").manual_seed(3)
    x, w = held8(300, K, g), held8(F, K, g)
    lin = B.Linear8(w, F, K, max_rows=300, stream=stream())
    full = torch.empty(300, F, device="cuda")
    lin.run(x, full, 300, stream=stream())
    size = x.double().abs() @ w.double().abs().t()
    for m in (1, 8, 9, 16, 17, 130, 299):
        y = torch.empty(m, F, device="cuda")
        lin.run(x, y, m, stream=stream())
        lin.check()
        assert ((y.double() - x[:m].double() @ w.double().t()).abs() <= (K / 32 + 10) * 2.0 ** -23 * size[:m]).all()
    lin.run(0, 0, 0)                                        # no rows: nothing to do
    refused(2, lin.run, x, full, 301)
    refused(2, lin.run, x, full, -1)
    refused(2, lin.run, x, full, 1, ldx=K - 1)
    refused(2, lin.run, x, full, 1, ldy=F - 1)
    refused(1, lin.run, 0, full, 1)
    refused(1, lin.run, x, 0, 1)
    refused(2, lin.run_mx8, 72, full, 1)
    refused(1, lin.run_mx8, 0, full, 1)
    refused(2, lin.debug_wait, 0, -1)


def test_another_stream_and_a_captured_graph():
    import torch
    from paper_2001_00138_b200 import binding as B
    M, K, F = 24, 1024, 512
    g = torch.Generator(device="cuda").manual_seed(4)
    xs = [torch.randn(M, K, generator=g, device="cuda") for _ in range(3)]
    w = torch.randn(F, K, generator=g, device="cuda")
    lin = B.Linear8(w, F, K, max_rows=M, stream=stream())
    wants = []
    for x in xs:
        y = torch.empty(M, F, device="cuda")
        lin.run(x, y, M, stream=stream())
        wants.append(y)
    torch.cuda.synchronize()
    side, x, y = torch.cuda.Stream(), torch.zeros(M, K, device="cuda"), torch.empty(M, F, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        x.copy_(xs[0])
        lin.run(x, y, M, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(y, wants[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lin.run(x, y, M, stream=torch.cuda.current_stream().cuda_stream)
    for v, want in zip(xs, wants):
        x.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_offsets_beyond_32_bits():
    """A matrix of more than 2^31 elements: quantised, read back, and multiplied; its first and last rows are looked at."""
    import torch
    from paper_2001_00138_b200 import binding as B
    rows, K, F = 2 ** 23 + 133, 256, 16
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, K, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, rows, 1 << 20):
        x[lo:lo + (1 << 20)].copy_(torch.randn(min(1 << 20, rows - lo), K, generator=g, device="cuda"))
    w = torch.randn(F, K, generator=g, device="cuda").bfloat16()
    mx = torch.empty(B.mx8_bytes(rows, K), dtype=torch.uint8, device="cuda")
    back, y = torch.empty_like(x), torch.empty(rows, F, dtype=torch.bfloat16, device="cuda")
    B.mx8_quantize(x, mx, rows, K, dtype=B.BF16, stream=stream())
    B.mx8_dequantize(mx, back, rows, K, dtype=B.BF16, stream=stream())
    lin = B.Linear8(w, F, K, max_rows=0, dtype=B.BF16, stream=stream())
    lin.run_mx8(mx, y, rows, stream=stream())
    lin.check()
    wq = R.quantise8(w.double().cpu().numpy())
    for part in (slice(0, 200), slice(2 ** 23 - 70, 2 ** 23 + 133)):
        xq = R.quantise8(x[part].double().cpu().numpy())
        assert np.array_equal(back[part].double().cpu().numpy(), xq)
        ref = xq @ wq.T
        R.within(y[part].double().cpu().numpy(), ref, product_bound(K, np.abs(xq) @ np.abs(wq).T, ref, "bf16"), "y")


@pytest.mark.parametrize("rows", [3, 40])
def test_row_strides_beyond_32_bits(rows):
    import torch
    from paper_2001_00138_b200 import binding as B
    K, F = 300, 130
    ld = 2 ** 31 // (rows - 1) + 64
    g = torch.Generator().manual_seed(rows)
    x, w = torch.randn(rows, K, generator=g).half(), (torch.randn(F, K, generator=g) / 17).half()
    fx, fy = (torch.empty((rows - 1) * ld + n, dtype=torch.float16, device="cuda") for n in (K, F))
    xv, y = torch.as_strided(fx, (rows, K), (ld, 1)), torch.as_strided(fy, (rows, F), (ld, 1))
    xv.copy_(x)
    lin = B.Linear8(w.cuda(), F, K, max_rows=rows, dtype=B.F16, stream=stream())
    lin.run(xv, y, rows, ldx=ld, ldy=ld, stream=stream())
    lin.check()
    xq, wq = R.quantise8(x.double().numpy()), R.quantise8(w.double().numpy())
    ref = xq @ wq.T
    R.within(y.double().cpu().numpy(), ref, product_bound(K, np.abs(xq) @ np.abs(wq).T, ref, "f16"), "y")


@pytest.mark.parametrize("form, skip", [("quantises its rows, one tile", 1), ("quantises its rows, cluster of four", 2), ("a cluster of eight", 3),
                                        ("no cluster, ring wraps", 9), ("256 outputs, few of them", 7), ("256 outputs, ring wraps", 11)])
def test_a_wait_that_runs_out_is_reported_and_the_handle_keeps_working(form, skip):
    """The bound is shortened to a few milliseconds and the copies of one column tile are left out, so that the consumers' wait for them runs out."""
    import torch
    from paper_2001_00138_b200 import binding as B
    rows, K, F, mx, _ = FORMS[form]
    g = torch.Generator(device="cuda").manual_seed(0)
    x, w = (torch.randint(-4, 5, (n, K), generator=g, device="cuda").bfloat16() for n in (rows, F))
    y = torch.full((rows, F), float("nan"), dtype=torch.bfloat16, device="cuda")
    lin = B.Linear8(w, F, K, max_rows=rows, dtype=B.BF16, stream=stream())
    want = (x.double() @ w.double().t()).bfloat16()
    lin.run(x, y, rows, stream=stream())
    lin.check()
    assert torch.equal(y, want)
    lin.debug_wait(1024, skip)
    lin.run(x, y, rows, stream=stream())
    refused(E_DEVICE_TIMEOUT, lin.check)
    lin.check()                                            # the report cleared the status word
    lin.debug_wait(0, 0)
    y.fill_(float("nan"))
    lin.run(x, y, rows, stream=stream())
    lin.check()
    assert torch.equal(y, want)
