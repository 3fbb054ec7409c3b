"""4-bit microscaled matrices and the linear layer on them against 64-bit statements.

Quantised values are whole multiples of a power of two and have to be equal.  Products of them are exact in fp32; their sum is
accumulated 64 columns at a time, so it is off by at most (K / 64 + 8) roundings (counted as truncations, 2^-23) of sum |x| |w|, fixed
before the first run; the activation adds two roundings, and the output is rounded once.
"""
import numpy as np
import pytest

import ops_ref as R

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "silu"]


def types(dtype):
    import torch
    from paper_2001_00138_b200 import binding as B
    return {"f32": (torch.float32, B.F32), "f16": (torch.float16, B.F16), "bf16": (torch.bfloat16, B.BF16)}[dtype]


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def buffer(rows, cols, fill=255):
    """A 4-bit matrix's buffer full of codes and scales that are wrong (255 = NaN scales) where nothing writes them."""
    import torch
    from paper_2001_00138_b200 import binding as B
    return torch.full((max(16, B.mx4_bytes(rows, cols)),), fill, dtype=torch.uint8, device="cuda")


def spaced(v, slack, offset=0):
    import torch
    r, c = v.shape
    flat = torch.full((r * (c + slack) + 16,), float("nan"), dtype=v.dtype, device="cuda")
    view = torch.as_strided(flat, (r, c), (c + slack, 1), offset)
    view.copy_(v)
    return flat, view


SIZES = [(1, 1), (1, 31), (3, 32), (2, 33), (8, 63), (33, 64), (128, 65), (129, 128), (31, 129), (97, 200), (5, 256), (7, 257), (256, 1000), (130, 2049)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("slack", [0, 8, 3])
def test_quantise_and_back(rows, cols, dtype, slack):
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = types(dtype)
    g = torch.Generator().manual_seed(rows * 1000 + cols)
    x = (torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-6, 6, (rows, 1), generator=g).float())).to(tt)
    _, v = spaced(x, slack)
    mx = buffer(rows, cols)
    B.mx4_quantize(v, mx, rows, cols, dtype=dt, ld=v.stride(0), stream=stream())
    flat, out = spaced(torch.zeros(rows, cols, dtype=tt), slack)
    B.mx4_dequantize(mx, out, rows, cols, dtype=dt, ld=out.stride(0), stream=stream())
    torch.cuda.synchronize()
    assert np.array_equal(out.double().cpu().numpy(), R.quantise(x.double().numpy()))
    inside = torch.zeros_like(flat, dtype=torch.bool)
    torch.as_strided(inside, out.shape, out.stride()).fill_(True)
    assert torch.isnan(flat[~inside]).all()


def round_trip(x):
    import torch
    from paper_2001_00138_b200 import binding as B
    rows, cols = x.shape
    mx = buffer(rows, cols)
    out = torch.empty(rows, cols, device="cuda")
    B.mx4_quantize(x.cuda(), mx, rows, cols, stream=stream())
    B.mx4_dequantize(mx, out, rows, cols, stream=stream())
    torch.cuda.synchronize()
    return out.cpu().double().numpy()


def test_ties_saturation_signs_and_extreme_scales():
    import torch
    # every quarter step of the scaled range, at block maxima from just below 8 (scale 1: 7.9 becomes 6) to subnormals and the largest floats
    steps = torch.arange(-31, 32).float() / 4
    rows = []
    for top in (7.75, 4.0, 6.0, 5.0, 7.99):
        for base in (0, 16, 31):
            row = torch.cat([steps[base:base + 31].clamp(-top, top), torch.tensor([top])])
            rows.append(row)
    x = torch.stack(rows)
    assert np.array_equal(round_trip(x), R.quantise(x.double().numpy()))
    for e in (-149, -140, -128, -127, -126, -125, -60, 60, 124, 125):
        y = torch.ldexp(x.double(), torch.tensor(e)).float()
        y = y[torch.isfinite(y).all(1)]
        assert np.array_equal(round_trip(y), R.quantise(y.double().numpy())), e
    z = torch.zeros(4, 64)
    assert not round_trip(z).any()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_not_finite_blocks(bad):
    import torch
    x = torch.randn(40, 100, generator=torch.Generator().manual_seed(1))
    x[7, 40] = bad
    x[39, 99] = bad
    got, ref = round_trip(x), R.quantise(x.double().numpy())
    assert np.isnan(ref[7, 32:64]).all() and np.isnan(ref[39, 96:]).all() and np.isnan(ref).sum() == 36
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
    lin = B.Linear(wv, F, K, max_rows=M, dtype=dt, bias=b.cuda() if bias else None, act=[B.ACT_NONE, B.ACT_RELU, B.ACT_SILU][ACTS.index(act)],
                   ldw=wv.stride(0), stream=stream())
    if mx:
        buf = buffer(M, K)
        B.mx4_quantize(xv, buf, M, K, dtype=dt, ld=xv.stride(0), stream=stream())
        lin.run_mx4(buf, y, M, ldy=y.stride(0), stream=stream())
    else:
        lin.run(xv, y, M, ldx=xv.stride(0), ldy=y.stride(0), stream=stream())
    lin.check()
    xq, wq = R.quantise(x.double().numpy()), R.quantise(w.double().numpy())
    z = xq @ wq.T + (b.double().numpy() if bias else 0)
    ref = R.act(z, act)
    size = np.abs(xq) @ np.abs(wq).T + np.abs(b.double().numpy())
    bound = 1.1 * (K / 64 + 10) * 2.0 ** -23 * size + R.UNIT[dtype] * np.abs(ref) * 1.01 + R.TINY[dtype]
    R.within(y.double().cpu().numpy(), ref, bound, f"{M} x {K} x {F} {dtype} {act}")
    inside = torch.zeros_like(flat, dtype=torch.bool)
    torch.as_strided(inside, y.shape, y.stride()).fill_(True)
    assert torch.isnan(flat[~inside]).all()
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
def test_linear_strides_and_4_bit_rows(M, K, F, dtype, slack):
    linear_case(M, K, F, dtype, "relu", slack=slack, seed=5)
    linear_case(M, K, F, dtype, "silu", slack=slack, seed=6, mx=True)


@pytest.mark.parametrize("M", [1, 5, 40, 300])
def test_a_row_that_is_not_finite_spoils_no_other(M):
    import torch
    from paper_2001_00138_b200 import binding as B
    K, F = 600, 200
    g = torch.Generator().manual_seed(2)
    x, w = torch.randn(M, K, generator=g).cuda(), torch.randn(F, K, generator=g).cuda()
    lin = B.Linear(w, F, K, max_rows=M, stream=stream())
    y0, y1 = torch.empty(M, F, device="cuda"), torch.empty(M, F, device="cuda")
    lin.run(x, y0, M, stream=stream())
    x[M // 2, 333] = float("inf")
    lin.run(x, y1, M, stream=stream())
    lin.check()
    others = torch.arange(M, device="cuda") != M // 2
    assert torch.isnan(y1[M // 2]).all() and torch.isfinite(y0).all()
    assert torch.equal(y1[others], y0[others])


def test_fewer_rows_than_the_handle_was_made_for_and_refusals():
    import torch
    from paper_2001_00138_b200 import binding as B
    K, F = 384, 96
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn(300, K, generator=g).cuda(), torch.randn(F, K, generator=g).cuda()
    lin = B.Linear(w, F, K, max_rows=300, stream=stream())
    full = torch.empty(300, F, device="cuda")
    lin.run(x, full, 300, stream=stream())
    for m in (1, 16, 17, 130, 299):
        y = torch.empty(m, F, device="cuda")
        lin.run(x, y, m, stream=stream())
        lin.check()
        size = R.quantise(x[:m].double().cpu().numpy())
        size = np.abs(size) @ np.abs(R.quantise(w.double().cpu().numpy())).T
        R.within(y.double().cpu().numpy(), full[:m].double().cpu().numpy(), (K / 64 + 8) * 2.0 ** -22 * size, f"{m} rows")
    lin.run(0, 0, 0)                                        # no rows: nothing to do
    for status, call in ((2, lambda: lin.run(x, full, 301)), (2, lambda: lin.run(x, full, -1)), (2, lambda: lin.run(x, full, 1, ldx=K - 1)),
                         (2, lambda: lin.run(x, full, 1, ldy=F - 1)), (1, lambda: lin.run(0, full, 1)), (1, lambda: lin.run(x, 0, 1)),
                         (2, lambda: lin.run_mx4(72, full, 1)), (1, lambda: lin.run_mx4(0, full, 1))):
        with pytest.raises(B.PatdnnError) as e:
            call()
        assert e.value.status == status


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N, P, C, G, act, slack", [(1, 5, 20, 4, "none", 0), (2, 100, 64, 32, "relu", 0), (3, 77, 96, 8, "silu", 8), (1, 300, 320, 32, "relu", 3), (2, 30000, 64, 16, "silu", 0)])
def test_group_norm_into_4_bit_rows(N, P, C, G, act, slack, dtype):
    """The fused form equals quantising act(norm) in 64 bits except where rounding of the fp32 value decides between two neighbours: those
    elements (or, where it moves a block's largest value across a power of two, blocks) are few, and a neighbour away."""
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = types(dtype)
    g = torch.Generator().manual_seed(C)
    x = (torch.randn(N, P, C, generator=g) + torch.randn(C, generator=g)).to(tt)
    gamma, beta = 1 + 0.1 * torch.randn(C, generator=g), 0.1 * torch.randn(C, generator=g)
    _, xv = spaced(x.reshape(N * P, C), slack)
    h = B.GroupNorm(N, P, C, G, dtype=dt, act=[B.ACT_NONE, B.ACT_RELU, B.ACT_SILU][ACTS.index(act)], x_pixel=C + slack)
    mx, out, stats = buffer(N * P, C), torch.empty(N * P, C, device="cuda"), torch.empty(N, G, 2, device="cuda")
    h.run_mx4(xv, gamma.cuda(), beta.cuda(), mx, stats, stream())
    B.mx4_dequantize(mx, out, N * P, C, stream=stream())
    torch.cuda.synchronize()
    f = R.norm(x.double().numpy(), gamma.double().numpy(), beta.double().numpy(), G, 1e-5, act)
    want = R.quantise(f["y"].reshape(N * P, C))
    got = out.double().cpu().numpy()
    off = got != want
    assert off.mean() <= 1e-4, off.mean()
    size = np.abs(f["y"].reshape(N * P, C))
    block = np.stack([np.pad(size, ((0, 0), (0, -C % 32)))[:, i::32] for i in range(32)], -1).max(-1).repeat(32, axis=1)[:, :C]
    assert (np.abs(got - want) <= 0.5 * block).all()
    R.within(stats[..., 1].double().cpu().numpy(), f["rstd"], 64 * R.EPS24 * f["rstd"] * (1 + np.abs(f["mean"]) * f["rstd"]), "rstd")


def test_another_stream_and_a_captured_graph():
    import torch
    from paper_2001_00138_b200 import binding as B
    M, K, F = 24, 1024, 512
    g = torch.Generator().manual_seed(4)
    xs = [torch.randn(M, K, generator=g).cuda() for _ in range(3)]
    w = torch.randn(F, K, generator=g).cuda()
    lin = B.Linear(w, F, K, max_rows=M, stream=stream())
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
    for lo in range(0, rows, 1 << 20):                      # in pieces: the generator's fp32 values are never all there at once
        x[lo:lo + (1 << 20)].copy_(torch.randn(min(1 << 20, rows - lo), K, generator=g, device="cuda"))
    w = torch.randn(F, K, generator=g, device="cuda").bfloat16()
    mx = torch.empty(B.mx4_bytes(rows, K), dtype=torch.uint8, device="cuda")
    back, y = torch.empty_like(x), torch.empty(rows, F, dtype=torch.bfloat16, device="cuda")
    B.mx4_quantize(x, mx, rows, K, dtype=B.BF16, stream=stream())
    B.mx4_dequantize(mx, back, rows, K, dtype=B.BF16, stream=stream())
    lin = B.Linear(w, F, K, max_rows=0, dtype=B.BF16, stream=stream())
    lin.run_mx4(mx, y, rows, stream=stream())
    lin.check()
    wq = R.quantise(w.double().cpu().numpy())
    for part in (slice(0, 200), slice(2 ** 23 - 70, 2 ** 23 + 133)):
        xq = R.quantise(x[part].double().cpu().numpy())
        assert np.array_equal(back[part].double().cpu().numpy(), xq)
        ref = xq @ wq.T
        R.within(y[part].double().cpu().numpy(), ref, 14 * 2.0 ** -23 * (np.abs(xq) @ np.abs(wq).T) + R.UNIT["bf16"] * np.abs(ref) * 1.01 + R.TINY["bf16"], "y")


@pytest.mark.parametrize("rows", [3, 40])
def test_row_strides_beyond_32_bits(rows):
    """Rows so far apart that the last ones lie beyond 2^31 elements, for the kernel that quantises few rows itself and for two launches."""
    import torch
    from paper_2001_00138_b200 import binding as B
    K, F = 300, 130
    ld = 2 ** 31 // (rows - 1) + 64
    g = torch.Generator().manual_seed(rows)
    x, w = torch.randn(rows, K, generator=g).half(), (torch.randn(F, K, generator=g) / 17).half()
    fx, fy = (torch.empty((rows - 1) * ld + n, dtype=torch.float16, device="cuda") for n in (K, F))
    xv, y = torch.as_strided(fx, (rows, K), (ld, 1)), torch.as_strided(fy, (rows, F), (ld, 1))
    xv.copy_(x)
    lin = B.Linear(w.cuda(), F, K, max_rows=rows, dtype=B.F16, stream=stream())
    lin.run(xv, y, rows, ldx=ld, ldy=ld, stream=stream())
    lin.check()
    xq, wq = R.quantise(x.double().numpy()), R.quantise(w.double().numpy())
    ref = xq @ wq.T
    R.within(y.double().cpu().numpy(), ref, 15 * 2.0 ** -23 * (np.abs(xq) @ np.abs(wq).T) + R.UNIT["f16"] * np.abs(ref) * 1.01 + R.TINY["f16"], "y")
