"""Gradient of the gated block in half precision where dg = dh u act'(g) and du = dh act(g) leave half's range although the inputs and the gradients do not.

dg and du are rounded as operands of the products: at most 2^-11 of each, and half a step of half's smallest, 2^-25, where the largest of a row (dx) or
of a column (dwg, dwu) is between 2^-3 and 2^15; any other is brought between 2^14 and 2^15, where that is 2^-25 / 2^14 = 2^-39 of the largest.  The rest of the bounds is test_gpu_gated's: 8
roundings of fp32 in front, the products' fp32 sums, one rounding of the result.  Fixed before the first run.
"""
import pytest

import ff_ref as R
from ff_ref import stream, untouched
from test_gpu_gated import ACTS, Case, act, same, slope

pytestmark = pytest.mark.gpu


def bounds(c, name):
    """64-bit gradients of the case, and how far each may be off."""
    import torch
    x, wg, wu, dh = (t.double() for t in (c.x, c.wg, c.wu, c.dh))
    g, u = c.gu[:, 0].double(), c.gu[:, 1].double()
    dg, du = dh * u * slope(g, name), dh * act(g, name)
    unit = R.UNIT["f16"] * 1.01 + 8 * R.EPS24
    extra = 8 * R.EPS24 * (dh * u).abs() if name == "silu" else torch.zeros_like(dg)       # SiLU's slope near its zero

    def least(top):                                        # (a largest one next to a border may fall on either side of it: the larger of the two)
        return torch.where((top > 2.0 ** -3 * 0.999) & (top < 2.0 ** 15 * 1.001), torch.clamp_min(top * 2.0 ** -39, 2.0 ** -25), top * 2.0 ** -39)

    row = least(torch.maximum(dg.abs().amax(1, keepdim=True), du.abs().amax(1, keepdim=True)))
    og, ou = unit * dg.abs() + extra + row, unit * du.abs() + row
    dx, size = dg @ wg + du @ wu, dg.abs() @ wg.abs() + du.abs() @ wu.abs()
    yield "dx", c.dx, dx, og @ wg.abs() + ou @ wu.abs() + (2 * c.F / 16 + 14) * 2.0 ** -23 * size
    for what, got, d, more in (("dwg", c.dwg, dg, extra), ("dwu", c.dwu, du, 0)):
        off = unit * d.abs() + more + least(d.abs().amax(0, keepdim=True))
        yield what, got, d.t() @ x, off.t() @ x.abs() + (c.M / 16 + 14) * 2.0 ** -23 * (d.abs().t() @ x.abs())


def check(c, name):
    import torch
    c.backward()
    for what, got, want, bound in bounds(c, name):
        assert want.abs().max() < 65000 and torch.isfinite(got).all(), (what, want.abs().max().item(), int((~torch.isfinite(got)).sum()))
        bad = ~((got.double() - want).abs() <= bound + R.UNIT["f16"] * 1.01 * want.abs() + R.TINY["f16"])
        assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist(), bound[bad][:4].tolist())
    assert untouched(c.fdx, c.dx) and untouched(c.fdg, c.dwg) and untouched(c.fdu, c.dwu)


SIZES = [(1, 64, 8), (3, 100, 70), (40, 200, 333), (300, 136, 264), (777, 1000, 1333), (3000, 256, 300), (5000, 72, 2050)]


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("M, K, F", SIZES)
def test_large_products(M, K, F, name):
    """dh and u around 300: dg around 90000, above half's largest number; weights and x small."""
    import torch
    c = Case(M, K, F, "f16", name, False, slack=8, seed=1)
    g = torch.Generator(device="cuda").manual_seed(M)
    c.gu.copy_(torch.randn(c.gu.shape, generator=g, device="cuda") * torch.tensor([2.0, 300.0], device="cuda")[:, None])
    c.dh.mul_(300)
    c.wg.mul_(2.0 ** -10)
    c.wu.mul_(2.0 ** -5)
    c.x.mul_(2.0 ** -10)
    assert (c.dh.double() * c.gu[:, 1].double()).abs().max() > 65504 or M * F < 500
    check(c, name)


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("M, K, F", SIZES)
def test_small_products(M, K, F, name):
    """A mean loss that was not scaled: dh of 1e-5, g and u of 1e-3: du around 1e-8, below half's smallest number; weights, and thousands of rows, make up for it."""
    import torch
    c = Case(M, K, F, "f16", name, False, wslack=3, seed=2)
    g = torch.Generator(device="cuda").manual_seed(M)
    c.gu.copy_(torch.randn(c.gu.shape, generator=g, device="cuda") * 1e-3)
    c.dh.mul_(1e-5)
    c.wg.mul_(3000)
    c.wu.mul_(3000)
    c.x.mul_(3000)
    check(c, name)
    assert c.dx.any() and c.dwg.any() and c.dwu.any()


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("M, K, F", SIZES)
def test_rows_and_columns_of_very_different_magnitudes(M, K, F, name):
    """Rows of dh and columns of u from 2^-11 to 2^11, in one call; rows and columns without any gradient among them."""
    import torch
    c = Case(M, K, F, "f16", name, False, hslack=1, seed=3)
    g = torch.Generator(device="cuda").manual_seed(M)
    rows = torch.exp2(torch.randint(-11, 12, (M, 1), generator=g, device="cuda").float())
    cols = torch.exp2(torch.randint(-11, 12, (F,), generator=g, device="cuda").float())
    c.gu.copy_(torch.randn(c.gu.shape, generator=g, device="cuda"))
    c.gu[:, 1].copy_((c.gu[:, 1].float() * cols).half())
    c.dh.copy_((c.dh.float().clamp(-4, 4) * rows).half())
    c.wg.mul_(2.0 ** -9)
    c.wu.mul_(2.0 ** -9)
    c.x.mul_(2.0 ** -13)
    if M > 2:
        c.dh[M // 2] = 0
        c.gu[:, :, F // 2] = 0
    check(c, name)
    if M > 2:
        assert not c.dx[M // 2].any() and not c.dwg[F // 2].any() and not c.dwu[F // 2].any()


@pytest.mark.parametrize("dx, dw", [(True, False), (False, True)])
def test_whole_numbers_out_of_range(dx, dw):
    """dh and u whole multiples of 256, weights and x of 2^-12: dg up to 2^20, everything exact; one product at a time."""
    import torch
    for M, K, F in ((5, 72, 64), (300, 136, 333), (2500, 300, 700)):
        c = Case(M, K, F, "f16", "none", True, slack=3)
        gen = torch.Generator(device="cuda").manual_seed(1)
        c.gu.copy_(torch.randint(-4, 5, c.gu.shape, generator=gen, device="cuda") * 256)
        c.dh.mul_(256)
        for t in (c.x, c.wg, c.wu):
            t.mul_(2.0 ** -12)
        x, wg, wu, dh, g, u = (t.double() for t in (c.x, c.wg, c.wu, c.dh, c.gu[:, 0], c.gu[:, 1]))
        dg, du = dh * u, dh * g
        assert dg.abs().max() > 65504
        c.backward(dx, dw)
        wants = [dg @ wg + du @ wu, dg.t() @ x, du.t() @ x]
        assert max(t.abs().max() for t in wants) < 65000
        for got, want, asked in zip((c.dx, c.dwg, c.dwu), wants, (dx, dw, dw)):
            if asked:
                same(got, want.half().double(), (M, K, F))
            else:
                assert not got.any()
        assert untouched(c.fdx, c.dx)


def test_calls_of_one_handle_do_not_leave_magnitudes_behind():
    """A call with large values, then one with small ones, then fewer rows, in a captured graph too: each the bits of a fresh handle."""
    import torch
    from paper_2001_00138_b200 import binding as B
    M, K, F = 300, 136, 200
    c, fresh = Case(M, K, F, "f16", "silu", False), Case(M, K, F, "f16", "silu", False)
    c.forward()
    gu, dh = c.gu.clone(), c.dh.clone()

    def set_(scale):
        for one in (c, fresh):
            one.gu.copy_(gu)
            one.dh.copy_((dh.float() * scale).half())

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.block.grad(c.x, c.wg, c.wu, c.gu, c.dh, c.dx, c.dwg, c.dwu, M, stream=stream())
    for scale in (1000.0, 1e-4, 1.0):
        for rows in (M, 37):
            set_(scale)
            fresh.block.free()
            fresh.block = B.Gated(F, K, max_rows=M, dtype=B.F16, act=B.ACT_SILU, grad=True)
            c.M = fresh.M = rows
            c.backward()
            fresh.backward()
            assert torch.equal(c.dx[:rows], fresh.dx[:rows]) and torch.equal(c.dwg, fresh.dwg) and torch.equal(c.dwu, fresh.dwu), (scale, rows)
        c.M = fresh.M = M
        fresh.backward()
        for t in (c.dx, c.dwg, c.dwu):
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.dx, fresh.dx) and torch.equal(c.dwg, fresh.dwg) and torch.equal(c.dwu, fresh.dwu), scale


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("M, K, F", [(1, 64, 8), (40, 200, 333), (300, 136, 264)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_nothing_flows_through_a_stored_infinity_where_dh_or_the_slope_is_zero(M, K, F, dtype, name):
    """gu holds an infinity where g or u left the type's range: a number that is too large for it, whose product with a dh of 0 (a masked row, an output
    that nobody used), or with the slope of a shut gate, is 0 and not NaN.  Beside them everything is as with any finite number there."""
    import torch
    c = Case(M, K, F, dtype, name, False, seed=4)
    c.forward()
    g = torch.Generator(device="cuda").manual_seed(M)
    masked = torch.rand(M, F, generator=g, device="cuda") < 0.3
    shut = torch.rand(M, F, generator=g, device="cuda") < 0.2 if name != "none" else torch.zeros_like(masked)
    c.dh.masked_fill_(masked, 0)
    gate, up = c.gu[:, 0], c.gu[:, 1]
    if name != "none":
        gate.masked_fill_(shut, float("-inf"))
    c.backward()
    want = [t.clone() for t in (c.dx, c.dwg, c.dwu)]
    assert all(torch.isfinite(t).all() for t in want)
    sign = torch.where(torch.rand(M, F, generator=g, device="cuda") < 0.5, 1.0, -1.0)
    up.copy_(torch.where(masked | shut, sign * float("inf"), up.float()))
    gate.copy_(torch.where(masked & ~shut, sign * float("inf"), gate.float()))
    c.backward()
    for got, w in zip((c.dx, c.dwg, c.dwu), want):
        assert torch.equal(got, w)
    # whatever else a masked place holds
    up.masked_fill_(masked, float("nan"))
    gate.masked_fill_(masked, float("nan"))
    c.backward()
    for got, w in zip((c.dx, c.dwg, c.dwu), want):
        assert torch.equal(got, w)
    # a NaN that a gradient reaches: its row of dx and its row of dwg are NaN, others are as before
    up[M // 2, F // 3], gate[M // 2, F // 3], c.dh[M // 2, F // 3] = float("nan"), 1.0, 1.0
    c.backward()
    rows, cols = torch.arange(M, device="cuda") != M // 2, torch.arange(F, device="cuda") != F // 3
    assert torch.isnan(c.dwg[F // 3]).all() and torch.isnan(c.dx[M // 2]).all() and torch.isfinite(c.dwu).all()
    assert torch.equal(c.dx[rows], want[0][rows]) and torch.equal(c.dwg[cols], want[1][cols]) and torch.equal(c.dwu[cols], want[2][cols])
