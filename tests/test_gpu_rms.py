"""RMS norm with the residual's addition, its 8-bit form and its gradient against 64-bit statements.

Roundings, counted as 2^-24 each before the first run: s has one; a sum of C squares at most ADDS = 40 + 8 C / 8192 additions on its longest
way (16 in a lane, 5 in a warp, one per warp), each square two for s and one of its own; the mean, the sum with eps, the root and the
reciprocal one each, half of them behind the root: rstd is off by (ADDS + 8) / 2 of them, y by that, s's one and two products, then its own.
"""
import numpy as np
import pytest

import ff_ref as R
from ff_ref import refused, spaced, stream, types, untouched

pytestmark = pytest.mark.gpu
EPS = 1e-5


def adds(C):
    return 40 + 8 * C / 8192


def case(M, C, dtype, slack, seed, offset=0):
    import torch
    tt, dt = types(dtype)
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(M, C, generator=g, device="cuda") * torch.exp2(torch.randint(-6, 7, (M, 1), generator=g, device="cuda").float())).to(tt)
    r = (torch.randn(M, C, generator=g, device="cuda") * 2).to(tt)
    gamma = 1 + 0.3 * torch.randn(C, generator=g, device="cuda")
    return tt, dt, spaced(x, slack, offset), spaced(r, slack, offset), gamma


def check(got, ref, bound, what):
    bad = ~((got.double() - ref).abs() <= bound)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:3].tolist(), got.double()[bad][:3].tolist(), ref[bad][:3].tolist(), bound[bad][:3].tolist())


def forward_reference(x, r, gamma):
    s = x.double() + (0 if r is None else r.double())
    rstd = ((s * s).mean(1, keepdim=True) + EPS) ** -0.5
    return s, rstd, s * rstd * gamma.double()


SIZES = [(5001, 36), (3002, 100), (2999, 7), (70, 64), (700, 65), (333, 2560), (1, 1), (1, 8), (3, 31), (2, 127), (5, 128), (4, 129), (40, 256), (33, 257), (7, 1000), (1, 4096), (300, 1001), (3000, 512), (200, 2050), (700, 4096), (5, 5000),
         (260, 8192), (3, 8193), (170, 12345), (2, 16384), (40, 20001), (3, 65536)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M, C", SIZES)
@pytest.mark.parametrize("slack, offset", [(0, 0), (8, 8), (2, 2), (3, 1)])
def test_forward(M, C, dtype, slack, offset):
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt, (_, x), (_, r), gamma = case(M, C, dtype, slack, M + C, offset)
    h = B.RmsNorm(C, dtype=dt, eps=EPS, x_row=C + slack, r_row=C + slack, y_row=C + slack)
    fs, total = spaced(torch.zeros(M, C, dtype=tt), slack, offset)
    fy, y = spaced(torch.zeros(M, C, dtype=tt), slack, offset)
    rstd = torch.full((M,), float("nan"), device="cuda")
    h.run(x, gamma, y, M, residual=r, sum=total, rstd=rstd, stream=stream())
    torch.cuda.synchronize()
    s, rs, want = forward_reference(x, r, gamma)
    check(total, s, (R.EPS24 + R.UNIT[dtype] * 1.01) * s.abs() + R.TINY[dtype], "sum")
    check(rstd[:, None], rs, (adds(C) + 8) / 2 * R.EPS24 * rs * 1.01, "rstd")
    check(y, want, ((adds(C) + 8) / 2 + 3) * 1.01 * R.EPS24 * want.abs() + R.UNIT[dtype] * 1.01 * want.abs() + R.TINY[dtype], "y")
    assert untouched(fs, total) and untouched(fy, y)
    # without a residual, without outputs that nobody asked for; the same bits where nothing else differs
    y2 = torch.full_like(fy, float("nan"))
    y2 = torch.as_strided(y2, y.shape, y.stride(), offset)
    h.run(x, gamma, y2, M, stream=stream())
    torch.cuda.synchronize()
    s, rs, want = forward_reference(x, None, gamma)
    check(y2, want, ((adds(C) + 8) / 2 + 3) * 1.01 * R.EPS24 * want.abs() + R.UNIT[dtype] * 1.01 * want.abs() + R.TINY[dtype], "y alone")
    # the sum in the residual's place
    y3 = torch.full_like(y, float("nan")) if slack == 0 else torch.as_strided(torch.full_like(fy, float("nan")), y.shape, y.stride(), offset)
    h.run(x, gamma, y3, M, residual=r, sum=r, stream=stream())
    torch.cuda.synchronize()
    assert torch.equal(y3, y) and torch.equal(r, total)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M, C", [(5001, 36), (3002, 100), (2999, 7), (200, 2560), (1, 1), (3, 31), (40, 127), (130, 128), (257, 129), (33, 1000), (1, 4096), (500, 2048), (9, 5001), (300, 8192), (140, 9000), (3, 65536)])
@pytest.mark.parametrize("slack", [0, 8, 2, 3])
def test_8_bit_form(M, C, dtype, slack):
    """Equal to the quantisation (tested by itself) of the fp32 values that the formula gives step by step with the statistics that the call returns."""
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt, (_, x), (_, r), gamma = case(M, C, dtype, slack, M * 3 + C)
    h = B.RmsNorm(C, dtype=dt, eps=EPS, x_row=C + slack, r_row=C + slack)
    mx, again, rstd = R.mx8_buffer(M, C), R.mx8_buffer(M, C), torch.full((M,), float("nan"), device="cuda")
    _, total = spaced(torch.zeros(M, C, dtype=tt), slack)
    h.run_mx8(x, gamma, mx, M, residual=r, sum=total, rstd=rstd, stream=stream())
    z = (x.float() + r.float()) * rstd[:, None] * gamma
    B.mx8_quantize(z, again, M, C, stream=stream())
    a, b = torch.empty(M, C, device="cuda"), torch.empty(M, C, device="cuda")
    B.mx8_dequantize(mx, a, M, C, stream=stream())
    B.mx8_dequantize(again, b, M, C, stream=stream())
    torch.cuda.synchronize()
    s, rs, _ = forward_reference(x, r, gamma)
    check(rstd[:, None], rs, (adds(C) + 8) / 2 * R.EPS24 * rs * 1.01, "rstd")
    check(total, s, (R.EPS24 + R.UNIT[dtype] * 1.01) * s.abs() + R.TINY[dtype], "sum")
    assert torch.equal(a, b)


def gradient_reference(s, gamma, rstd, dy, ds):
    s, gamma, rstd, dy = s.double(), gamma.double(), rstd.double()[:, None], dy.double()
    xh, u = s * rstd, dy * gamma
    m = (u * xh).mean(1, keepdim=True)
    dx = rstd * (u - xh * m) + (0 if ds is None else ds.double())
    return dx, xh, u, m


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M, C", SIZES)
@pytest.mark.parametrize("slack, offset", [(0, 0), (8, 8), (2, 2), (3, 1)])
def test_gradient(M, C, dtype, slack, offset):
    """dx: u, xh and their product with the mean have 3 roundings, the mean (ADDS + 4) of the mean magnitude, three more behind; dgamma: at most
    M / 18 + 80 additions on the longest way (15 clusters at least share the rows of the longest rows: M / 15 + 15, less than that up to 5000 rows)."""
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt, (_, s), (_, dy), gamma = case(M, C, dtype, slack, M + 2 * C, offset)
    g = torch.Generator(device="cuda").manual_seed(7)
    _, ds = spaced(torch.randn(M, C, generator=g, device="cuda").to(tt), slack, offset)
    rstd = ((s.double() ** 2).mean(1) + EPS).rsqrt().float()
    h = B.RmsNorm(C, dtype=dt, eps=EPS, x_row=C + slack, r_row=C + slack, y_row=C + slack)
    f, dx = spaced(torch.zeros(M, C, dtype=tt), slack, offset)
    dgamma = torch.full((C,), float("nan"), device="cuda")
    for add in (ds, None):
        h.grad(s, gamma, rstd, dy, dx, dgamma, M, dsum=add, stream=stream())
        torch.cuda.synchronize()
        want, xh, u, m = gradient_reference(s, gamma, rstd, dy, add)
        rs = rstd.double()[:, None]
        size = rs * (u.abs() * 3 + xh.abs() * (m.abs() * 4 + (u * xh).abs().mean(1, keepdim=True) * (adds(C) + 4))) + want.abs() * 2
        check(dx, want, 1.01 * R.EPS24 * size + R.UNIT[dtype] * 1.01 * want.abs() + R.TINY[dtype], "dx")
        bound = (M / 18 + 80) * R.EPS24 * (dy.double() * xh).abs().sum(0)
        check(dgamma, (dy.double() * xh).sum(0), bound, "dgamma")
        assert untouched(f, dx)
    # in the place of dsum, of dy and of s
    h.grad(s, gamma, rstd, dy, dx, dgamma, M, dsum=ds, stream=stream())
    torch.cuda.synchronize()
    for place in (ds, dy, s):
        kept = place.clone()
        again = torch.full_like(dgamma, float("nan"))
        h.grad(s, gamma, rstd, dy, place, again, M, dsum=ds, stream=stream())
        torch.cuda.synchronize()
        assert torch.equal(place, dx) and torch.equal(again, dgamma)
        place.copy_(kept)


def test_gradient_against_differences():
    """fp32, a scalar of the outputs: central differences of the forward pass (step 2^-7: their own error is below 2^-12 of the scale)."""
    import torch
    from paper_2001_00138_b200 import binding as B
    M, C = 6, 300
    g = torch.Generator(device="cuda").manual_seed(0)
    x, r, a, b, vx, vg = (torch.randn(*s, generator=g, device="cuda") for s in ((M, C), (M, C), (M, C), (M, C), (M, C), (C,)))
    gamma = 1 + 0.3 * torch.randn(C, generator=g, device="cuda")
    h = B.RmsNorm(C, eps=EPS)
    y, total, rstd, dx, dgamma = torch.empty(M, C, device="cuda"), torch.empty(M, C, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, C, device="cuda"), torch.empty(C, device="cuda")

    def value(t):
        h.run(x + t * vx, gamma + t * vg, y, M, residual=r, sum=total, rstd=rstd, stream=stream())
        torch.cuda.synchronize()
        return ((y.double() * a.double()).sum() + (total.double() * b.double()).sum()).item()

    step = 2.0 ** -7
    slope = (value(step) - value(-step)) / (2 * step)
    value(0.0)
    h.grad(total, gamma, rstd, a, dx, dgamma, M, dsum=b, stream=stream())
    torch.cuda.synchronize()
    want = ((dx.double() * vx.double()).sum() + (dgamma.double() * vg.double()).sum()).item()
    scale = ((dx.double() * vx.double()).abs().sum() + (dgamma.double() * vg.double()).abs().sum()).item()
    assert abs(slope - want) < 2.0 ** -12 * scale, (slope, want, scale)


@pytest.mark.parametrize("M, C", [(1, 4096), (40, 4096), (40, 100), (12, 20000)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_row_that_is_not_finite_spoils_no_other(M, C, bad):
    import torch
    from paper_2001_00138_b200 import binding as B
    _, _, (_, x), (_, r), gamma = case(M, C, "f32", 0, 3)
    h = B.RmsNorm(C, eps=EPS)
    y0, y1 = torch.empty(M, C, device="cuda"), torch.empty(M, C, device="cuda")
    h.run(x, gamma, y0, M, residual=r, stream=stream())
    x[M // 2, C // 3] = bad
    h.run(x, gamma, y1, M, residual=r, stream=stream())
    mx = R.mx8_buffer(M, C)
    h.run_mx8(x, gamma, mx, M, residual=r, stream=stream())
    v = torch.empty(M, C, device="cuda")
    B.mx8_dequantize(mx, v, M, C, stream=stream())
    torch.cuda.synchronize()
    others = torch.arange(M, device="cuda") != M // 2
    if bad == bad:                                         # an infinity: s / inf = 0 in the other columns, NaN in its own
        assert torch.isnan(y1[M // 2, C // 3]) and (y1[M // 2].nan_to_num(0) == 0).all()
    else:
        assert torch.isnan(y1[M // 2]).all() and torch.isnan(v[M // 2]).all()
    assert torch.equal(y1[others], y0[others]) and torch.isfinite(v[others]).all()


def test_zero_rows_zeros_and_extreme_values():
    import torch
    from paper_2001_00138_b200 import binding as B
    C = 640
    h = B.RmsNorm(C, dtype=B.BF16, eps=EPS)
    gamma, dgamma = torch.ones(C, device="cuda"), torch.full((C,), float("nan"), device="cuda")
    h.run(0, 0, 0, 0)
    h.run_mx8(0, 0, 0, 0)
    h.grad(0, 0, 0, 0, 0, dgamma, 0, stream=stream())
    torch.cuda.synchronize()
    assert not dgamma.any()
    x = torch.zeros(3, C, dtype=torch.bfloat16, device="cuda")
    x[1] = 2.0 ** 60                                       # squares up to 2^120, their sum within range
    x[2] = 2.0 ** -120                                     # squares vanish beside eps
    y = torch.full_like(x, float("nan"))
    rstd = torch.empty(3, device="cuda")
    h.run(x, gamma, y, 3, rstd=rstd, stream=stream())
    torch.cuda.synchronize()
    assert not y[0].any() and (y[1] == 1).all() and torch.isfinite(y[2]).all()
    assert abs(rstd[0].item() * EPS ** 0.5 - 1) < 1e-6


def test_many_rows_and_offsets_beyond_32_bits():
    import torch
    from paper_2001_00138_b200 import binding as B
    M, C, ld = 40, 300, 2 ** 31 // 39 + 64
    g = torch.Generator(device="cuda").manual_seed(5)
    big = [torch.zeros((M - 1) * ld + C, dtype=torch.float16, device="cuda") for _ in range(4)]
    x, r, s, y = (torch.as_strided(b, (M, C), (ld, 1)) for b in big)
    x.copy_(torch.randn(M, C, generator=g, device="cuda"))
    r.copy_(torch.randn(M, C, generator=g, device="cuda"))
    gamma, rstd, dgamma = torch.ones(C, device="cuda"), torch.empty(M, device="cuda"), torch.empty(C, device="cuda")
    h = B.RmsNorm(C, dtype=B.F16, eps=EPS, x_row=ld, r_row=ld, y_row=ld)
    h.run(x, gamma, y, M, residual=r, sum=s, rstd=rstd, stream=stream())
    torch.cuda.synchronize()
    _, _, want = forward_reference(x, r, gamma)
    check(y, want, (40 * R.EPS24 + R.UNIT["f16"]) * 1.01 * want.abs() + R.TINY["f16"], "y")
    h.grad(s, gamma, rstd, y, x, dgamma, M, stream=stream())
    torch.cuda.synchronize()
    want, xh, u, m = gradient_reference(s, gamma, rstd, y, None)
    size = rstd.double()[:, None] * (u.abs() * 3 + xh.abs() * (m.abs() * 4 + (u * xh).abs().mean(1, keepdim=True) * 50)) + want.abs() * 2
    check(x, want, 1.01 * R.EPS24 * size + R.UNIT["f16"] * 1.01 * want.abs() + R.TINY["f16"], "dx")


def test_another_stream_and_captured_graphs():
    import torch
    from paper_2001_00138_b200 import binding as B
    M, C = 50, 768
    _, dt, _, _, gamma = case(M, C, "bf16", 0, 1)
    ins = [case(M, C, "bf16", 0, i)[2:4] for i in range(3)]
    h = B.RmsNorm(C, dtype=dt, eps=EPS)

    def passes(x, r, st):
        y, s, rstd, dx, dg = torch.empty_like(x), torch.empty_like(x), torch.empty(M, device="cuda"), torch.empty_like(x), torch.empty(C, device="cuda")
        h.run(x, gamma, y, M, residual=r, sum=s, rstd=rstd, stream=st)
        h.grad(s, gamma, rstd, y, dx, dg, M, dsum=r, stream=st)
        return y, s, rstd, dx, dg

    wants = [passes(x, r, stream()) for (_, x), (_, r) in ins]
    torch.cuda.synchronize()
    x, r = torch.zeros_like(ins[0][0][1]), torch.zeros_like(ins[0][0][1])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        x.copy_(ins[0][0][1])
        r.copy_(ins[0][1][1])
        got = passes(x, r, side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, wants[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = passes(x, r, torch.cuda.current_stream().cuda_stream)
    for ((_, a), (_, b)), want in zip(ins, wants):
        x.copy_(a)
        r.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_refusals_of_calls():
    import torch
    from paper_2001_00138_b200 import binding as B
    h = B.RmsNorm(64, dtype=B.F16)
    ok = torch.zeros(64, 64, device="cuda")
    p = ok.data_ptr()
    refused(2, h.run, ok, ok, ok, -1)
    refused(2, h.run, ok, ok, ok, 2 ** 31)
    refused(1, h.run, 0, ok, ok, 1)
    refused(1, h.run, ok, 0, ok, 1)
    refused(1, h.run, ok, ok, 0, 1)
    refused(2, h.run, p + 1, ok, ok, 1)
    refused(2, h.run, ok, p + 2, ok, 1)
    refused(2, h.run, ok, ok, p + 1, 1)
    refused(2, h.run, ok, ok, ok, 1, residual=p + 1)
    refused(2, h.run, ok, ok, ok, 1, sum=p + 1)
    refused(2, h.run, ok, ok, ok, 1, rstd=p + 2)
    refused(2, h.run_mx8, ok, ok, p + 8, 1)
    refused(1, h.grad, ok, ok, ok, ok, ok, 0, 1)
    for i in range(5):
        args = [ok] * 5
        args[i] = 0
        refused(1, h.grad, *args, ok, 1)
    refused(2, h.grad, ok, ok, ok, ok, p + 1, ok, 1)
    refused(2, h.grad, ok, ok, ok, ok, ok, p + 2, 1)
    refused(2, h.grad, ok, ok, ok, ok, ok, ok, 1, dsum=p + 1)


@pytest.mark.parametrize("C", [100, 640, 20000])
def test_rows_whose_squares_leave_the_range_of_fp32(C):
    """Magnitudes from 2^-140 to 2^126, eps = 0 and 1e-30: the same bound as elsewhere, on rows whose 1 / rms is a normal number."""
    import torch
    from paper_2001_00138_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(C)
    powers = [-120, -100, -80, -70, -60, -45, -40, -30, 0, 50, 56, 57, 60, 62, 64, 70, 100, 120]
    x = torch.ldexp(torch.rand(len(powers), C, generator=g, device="cuda") + 0.5, torch.tensor(powers, device="cuda")[:, None])
    gamma = 1 + 0.3 * torch.randn(C, generator=g, device="cuda")
    for eps in (0.0, 1e-30, 1e-6):
        h = B.RmsNorm(C, eps=eps)
        y, rstd = torch.empty_like(x), torch.empty(len(powers), device="cuda")
        h.run(x, gamma, y, len(powers), rstd=rstd, stream=stream())
        torch.cuda.synchronize()
        rs = ((x.double() ** 2).mean(1, keepdim=True) + float(np.float32(eps))) ** -0.5
        check(rstd[:, None], rs, (adds(C) + 8) / 2 * R.EPS24 * rs * 1.01, "rstd")
        want = x.double() * rs * gamma.double()
        check(y, want, ((adds(C) + 8) / 2 + 4) * 1.01 * R.EPS24 * want.abs() + R.TINY["f32"], "y")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_gradient_of_rows_of_every_length(dtype):
    """Every number of warps to a row, for rows one by one and for many; against the formula, with the bounds of test_gradient."""
    import torch
    from paper_2001_00138_b200 import binding as B
    for M in (60, 700):
        for C in [256 * w - 116 for w in range(1, 17)] + [512 * w - 31 for w in range(9, 17)] + [33000]:
            tt, dt, (_, s), (_, dy), gamma = case(M, C, dtype, 0, M + C)
            ds = torch.ones(M, C, device="cuda", dtype=tt)
            rstd = ((s.double() ** 2).mean(1) + EPS).rsqrt().float()
            dx, dgamma = torch.empty_like(s), torch.empty(C, device="cuda")
            B.RmsNorm(C, dtype=dt, eps=EPS).grad(s, gamma, rstd, dy, dx, dgamma, M, dsum=ds, stream=stream())
            torch.cuda.synchronize()
            want, xh, u, m = gradient_reference(s, gamma, rstd, dy, ds)
            rs = rstd.double()[:, None]
            size = rs * (u.abs() * 3 + xh.abs() * (m.abs() * 4 + (u * xh).abs().mean(1, keepdim=True) * (adds(C) + 4))) + want.abs() * 2
            check(dx, want, 1.01 * R.EPS24 * size + R.UNIT[dtype] * 1.01 * want.abs() + R.TINY[dtype], f"dx {M} x {C}")
            check(dgamma, (dy.double() * xh).sum(0), (M / 18 + 80) * R.EPS24 * (dy.double() * xh).abs().sum(0), f"dgamma {M} x {C}")


@pytest.mark.parametrize("M, C", [(1500, 9000), (700, 20008), (300, 40001)])
def test_long_rows_many_times_over(M, C):
    """Clusters of two, four and eight CTAs that exchange sums for many rows; the same bits from the same call, alone and beside another stream's."""
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt, (_, x), (_, r), gamma = case(M, C, "bf16", 0, M + C)
    h, other = B.RmsNorm(C, dtype=dt, eps=EPS), B.RmsNorm(C, dtype=dt, eps=EPS)
    total, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(M, device="cuda")
    h.run(x, gamma, y, M, residual=r, sum=total, rstd=rstd, stream=stream())
    torch.cuda.synchronize()
    s, rs, want = forward_reference(x, r, gamma)
    check(rstd[:, None], rs, (adds(C) + 8) / 2 * R.EPS24 * rs * 1.01, "rstd")
    check(y, want, ((adds(C) + 8) / 2 + 3) * 1.01 * R.EPS24 * want.abs() + R.UNIT["bf16"] * 1.01 * want.abs() + R.TINY["bf16"], "y")
    dx, dgamma = torch.empty_like(x), torch.empty(C, device="cuda")
    h.grad(total, gamma, rstd, r, dx, dgamma, M, dsum=x, stream=stream())
    torch.cuda.synchronize()
    want, xh, u, m = gradient_reference(total, gamma, rstd, r, x)
    rs = rstd.double()[:, None]
    size = rs * (u.abs() * 3 + xh.abs() * (m.abs() * 4 + (u * xh).abs().mean(1, keepdim=True) * (adds(C) + 4))) + want.abs() * 2
    check(dx, want, 1.01 * R.EPS24 * size + R.UNIT["bf16"] * 1.01 * want.abs() + R.TINY["bf16"], "dx")
    check(dgamma, (r.double() * xh).sum(0), (M / 15 + 95) * R.EPS24 * (r.double() * xh).abs().sum(0), "dgamma")
    side = torch.cuda.Stream()
    y2, dx2, dgamma2, y3, dx3, dgamma3 = (torch.full_like(t, float("nan")) for t in (y, dx, dgamma, y, dx, dgamma))
    torch.cuda.synchronize()
    for _ in range(5):
        h.run(x, gamma, y2, M, residual=r, stream=stream())
        other.grad(total, gamma, rstd, r, dx3, dgamma3, M, dsum=x, stream=side.cuda_stream)
        h.grad(total, gamma, rstd, r, dx2, dgamma2, M, dsum=x, stream=stream())
        other.run(x, gamma, y3, M, residual=r, stream=side.cuda_stream)
    torch.cuda.synchronize()
    for a, b in ((y, y2), (y, y3), (dx, dx2), (dx, dx3), (dgamma, dgamma2), (dgamma, dgamma3)):
        assert torch.equal(a, b)
