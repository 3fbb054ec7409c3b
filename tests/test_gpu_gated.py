"""Gated feed-forward block and its gradients against 64-bit statements on the device.

Whole numbers: products and sums that fp32 holds exactly, so every output has to be the rounded exact value.  Random values: a product's fp32
sum, 16 columns at a time, is off by at most (K / 16 + 10) roundings (counted as truncations, 2^-23) of the sum of magnitudes; dg and du are
rounded to the type (UNIT, and 8 roundings of fp32 before that) as operands; the output is rounded once.  Fixed before the first run.
"""
import pytest

import ff_ref as R
from ff_ref import refused, spaced, stream, types, untouched

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "silu"]
E_NULL, E_SHAPE, E_DEVICE_TIMEOUT, E_SCRATCH = 1, 2, 8, 12


def act_of(name):
    from paper_2001_00138_b200 import binding as B
    return [B.ACT_NONE, B.ACT_RELU, B.ACT_SILU][ACTS.index(name)]


def act(z, name):
    import torch
    return z if name == "none" else z.clamp_min(0) if name == "relu" else z * torch.sigmoid(z)


def slope(z, name):
    import torch
    s = torch.sigmoid(z)
    return torch.ones_like(z) if name == "none" else (z > 0).to(z.dtype) if name == "relu" else s + z * s * (1 - s)


class Case:
    """Tensors of one block, rows `slack` apart."""

    def __init__(self, M, K, F, dtype, name, whole, slack=0, wslack=0, hslack=0, seed=0):
        import torch
        from paper_2001_00138_b200 import binding as B
        self.tt, dt = types(dtype)
        self.M, self.K, self.F, self.name, self.dtype = M, K, F, name, dtype
        g = torch.Generator(device="cuda").manual_seed(seed + M + K + F)

        def make(r, c, most, scale):
            if whole:                                      # mostly zeros where sums are long, so that they stay exact
                keep = torch.rand(r, c, generator=g, device="cuda") < min(1.0, 200.0 / max(K, F))
                return torch.randint(-most, most + 1, (r, c), generator=g, device="cuda") * keep
            return torch.randn(r, c, generator=g, device="cuda") * scale

        self.fx, self.x = spaced(make(M, K, 2, 1.0).to(self.tt), slack)
        self.fg, self.wg = spaced(make(F, K, 2, K ** -0.5).to(self.tt), wslack)
        self.fu, self.wu = spaced(make(F, K, 2, K ** -0.5).to(self.tt), wslack)
        self.fdh, self.dh = spaced((make(M, F, 3, 1.0) if not whole else torch.randint(-3, 4, (M, F), generator=g, device="cuda")).to(self.tt), hslack)
        self.fh, self.h = spaced(torch.zeros(M, F, dtype=self.tt), hslack)
        self.fdx, self.dx = spaced(torch.zeros(M, K, dtype=self.tt), slack)
        self.fdg, self.dwg = spaced(torch.zeros(F, K, dtype=self.tt), wslack)
        self.fdu, self.dwu = spaced(torch.zeros(F, K, dtype=self.tt), wslack)
        self.gu = torch.full((M, 2, F), float("nan"), dtype=self.tt, device="cuda")
        self.block = B.Gated(F, K, max_rows=M, dtype=dt, act=act_of(name), x_row=K + slack, w_row=K + wslack, h_row=F + hslack, grad=True)

    def forward(self, gu=True):
        self.block.run(self.x, self.wg, self.wu, self.h, self.M, gu=self.gu if gu else None, stream=stream())
        self.block.check()

    def backward(self, dx=True, dw=True):
        self.block.grad(self.x, self.wg, self.wu, self.gu, self.dh, self.dx if dx else None, self.dwg if dw else None, self.dwu if dw else None, self.M,
                        stream=stream())
        self.block.check()


def same(got, want, what):
    bad = got.double() != want
    assert not bad.any(), (what, int(bad.sum()), bad.numel(), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), want[bad][:4].tolist())


def exact_case(M, K, F, dtype, name, **kw):
    import torch
    c = Case(M, K, F, dtype, name, True, **kw)
    c.forward()
    x, wg, wu, dh = (t.double() for t in (c.x, c.wg, c.wu, c.dh))
    g, u = x @ wg.t(), x @ wu.t()
    assert max(g.abs().max(), u.abs().max()) < 2 ** 11 and (g.abs() * u.abs()).max() < 2 ** 24
    same(c.gu[:, 0], g.to(c.tt).double(), "g")
    same(c.gu[:, 1], u.to(c.tt).double(), "u")
    same(c.h, (act(g, name) * u).to(c.tt).double(), "h")
    assert untouched(c.fh, c.h)
    # the gradient: small whole numbers in gu, so that dg and du are exact in the type
    gen = torch.Generator(device="cuda").manual_seed(1)
    c.gu.copy_(torch.randint(-4, 5, c.gu.shape, generator=gen, device="cuda"))
    g, u = c.gu[:, 0].double(), c.gu[:, 1].double()
    c.backward()
    dg, du = dh * u * slope(g, name), dh * act(g, name)
    dx, dwg, dwu = dg @ wg + du @ wu, dg.t() @ x, du.t() @ x
    assert max(t.abs().max() for t in (dx, dwg, dwu)) < 2 ** 24
    same(c.dx, dx.to(c.tt).double(), "dx")
    same(c.dwg, dwg.to(c.tt).double(), "dwg")
    same(c.dwu, dwu.to(c.tt).double(), "dwu")
    assert untouched(c.fdx, c.dx) and untouched(c.fdg, c.dwg) and untouched(c.fdu, c.dwu)
    c.block.free()


SIZES = [(150, 20000, 256), (2500, 700, 2600), (200, 700, 70), (1, 4096, 100), (9, 2050, 1000), (40, 1024, 9999), (100, 3000, 40), (128, 8000, 520), (1, 1, 1), (1, 8, 8), (2, 64, 128), (3, 17, 5), (1, 512, 300), (7, 1000, 1333), (16, 256, 256), (65, 63, 65), (128, 128, 64), (129, 130, 129), (255, 520, 384), (256, 256, 128),
         (300, 1000, 1333), (513, 64, 1000), (1000, 2000, 136), (4000, 40, 24), (20000, 72, 100), (2500, 300, 700)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M, K, F", SIZES)
def test_whole_numbers(M, K, F, dtype):
    exact_case(M, K, F, dtype, ["none", "relu"][(M + K) % 2])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("slack, wslack, hslack", [(8, 0, 0), (0, 8, 8), (3, 0, 1), (0, 3, 0), (1, 1, 2), (2, 5, 3), (4, 4, 4), (7, 7, 7)])
@pytest.mark.parametrize("M, K, F", [(5, 200, 72), (300, 136, 333), (40, 65, 64), (290, 100, 60)])
def test_strides(M, K, F, dtype, slack, wslack, hslack):
    exact_case(M, K, F, dtype, "relu", slack=slack, wslack=wslack, hslack=hslack)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("M, K, F", [(1, 4096, 500), (33, 1000, 1333), (777, 1000, 1333), (1024, 512, 2048), (3000, 256, 300)])
def test_random_values(M, K, F, dtype, name):
    import torch
    c = Case(M, K, F, dtype, name, False, seed=3)
    c.forward()
    unit, tiny = R.UNIT[dtype], R.TINY[dtype]
    x, wg, wu, dh = (t.double() for t in (c.x, c.wg, c.wu, c.dh))

    def check(got, ref, bound, what):
        bad = ~((got.double() - ref).abs() <= bound + unit * 1.01 * ref.abs() + tiny)
        assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), ref[bad][:4].tolist(), bound[bad][:4].tolist())

    g, u = x @ wg.t(), x @ wu.t()
    eg, eu = ((K / 16 + 10) * 2.0 ** -23 * (x.abs() @ w.abs().t()) for w in (wg, wu))
    check(c.gu[:, 0], g, eg, "g")
    check(c.gu[:, 1], u, eu, "u")
    a = act(g, name)
    check(c.h, a * u, 1.1 * eg * (u.abs() + eu) + a.abs() * eu + 8 * R.EPS24 * (a * u).abs(), "h")
    g, u = c.gu[:, 0].double(), c.gu[:, 1].double()
    c.backward()
    dg, du = dh * u * slope(g, name), dh * act(g, name)
    # what dg and du are off by as operands; SiLU's slope is near zero around -1.28 and off by the roundings of its terms there
    og, ou = ((unit * 1.01 + 8 * R.EPS24) * t.abs() + tiny for t in (dg, du))
    if name == "silu":
        og = og + 8 * R.EPS24 * (dh * u).abs()
    size = dg.abs() @ wg.abs() + du.abs() @ wu.abs()
    check(c.dx, dg @ wg + du @ wu, og @ wg.abs() + ou @ wu.abs() + (2 * F / 16 + 14) * 2.0 ** -23 * size, "dx")
    for got, d, off, what in ((c.dwg, dg, og, "dwg"), (c.dwu, du, ou, "dwu")):
        check(got, d.t() @ x, off.t() @ x.abs() + (M / 16 + 14) * 2.0 ** -23 * (d.abs().t() @ x.abs()), what)


def test_gradient_against_differences():
    """fp16, the block as one function of x and both weights along a direction: central differences of the 64-bit function around the same point."""
    import torch
    M, K, F = 40, 200, 96
    c = Case(M, K, F, "f16", "silu", False, seed=9)
    c.forward()
    c.backward()
    g = torch.Generator(device="cuda").manual_seed(2)
    x, wg, wu, dh = (t.double() for t in (c.x, c.wg, c.wu, c.dh))
    for which, grad in (("x", c.dx), ("wg", c.dwg), ("wu", c.dwu)):
        v = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)

        def value(t):
            p = dict(x=x, wg=wg, wu=wu)
            p[which] = p[which] + t * v
            return (act(p["x"] @ p["wg"].t(), "silu") * (p["x"] @ p["wu"].t()) * dh).sum().item()

        got = (value(1e-5) - value(-1e-5)) / 2e-5
        want = (grad.double() * v).sum().item()
        scale = (grad.double() * v).abs().sum().item()
        assert abs(got - want) < 4 * 2.0 ** -11 * scale, (which, got, want, scale)     # gu, dg and du, and the gradients themselves in half


def test_the_parts_that_are_asked_for():
    import torch
    c = Case(300, 136, 200, "bf16", "silu", False)
    c.forward()
    h = c.h.clone()
    c.h.fill_(float("nan"))
    c.forward(gu=False)
    assert torch.equal(c.h, h)
    c.backward()
    want = [t.clone() for t in (c.dx, c.dwg, c.dwu)]
    for dx, dw in ((True, False), (False, True), (False, False)):
        for t in (c.dx, c.dwg, c.dwu):
            t.fill_(float("nan"))
        c.backward(dx, dw)
        for t, w, asked in zip((c.dx, c.dwg, c.dwu), want, (dx, dw, dw)):
            assert torch.equal(t, w) if asked else torch.isnan(t).all()


@pytest.mark.parametrize("M", [1, 5, 300])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_row_that_is_not_finite_spoils_no_other(M, bad):
    import torch
    c = Case(M, 200, 300, "bf16", "silu", False)
    c.forward()
    before = c.h.clone()
    c.x[M // 2, 77] = bad
    c.forward()
    others = torch.arange(M, device="cuda") != M // 2
    assert torch.equal(c.h[others], before[others]) and not torch.isfinite(c.h[M // 2]).any()


def test_fewer_rows_than_the_handle_was_made_for_and_none():
    import torch
    from paper_2001_00138_b200 import binding as B
    c = Case(600, 136, 264, "bf16", "relu", True, wslack=8)
    for m in (1, 2, 100, 257, 599):
        c.M = m
        c.h.fill_(7)
        c.dx.fill_(7)
        c.forward(gu=False)
        x = c.x[:m].double()
        same(c.h[:m], (act(x @ c.wg.double().t(), "relu") * (x @ c.wu.double().t())).to(c.tt).double(), m)
        gu = torch.randint(-4, 5, (m, 2, 264), device="cuda").to(c.tt)
        c.gu[:m] = gu
        c.backward()
        dh, g, u = c.dh[:m].double(), gu[:, 0].double(), gu[:, 1].double()
        dg, du = dh * u * slope(g, "relu"), dh * act(g, "relu")
        same(c.dx[:m], (dg @ c.wg.double() + du @ c.wu.double()).to(c.tt).double(), "dx")
        same(c.dwg, (dg.t() @ x).to(c.tt).double(), "dwg")
        same(c.dwu, (du.t() @ x).to(c.tt).double(), "dwu")
        assert (c.h[m:] == 7).all() and (c.dx[m:] == 7).all()
    c.block.run(0, 0, 0, 0, 0)
    c.M = 0
    c.backward()
    assert not c.dwg.any() and not c.dwu.any() and untouched(c.fdg, c.dwg) and untouched(c.fdu, c.dwu)


def test_another_stream_a_captured_graph_and_other_weights():
    import torch
    from paper_2001_00138_b200 import binding as B
    M, K, F = 70, 320, 200
    cases = [Case(M, K, F, "bf16", "silu", False, seed=s) for s in range(3)]
    for c in cases:
        c.forward()
        c.backward()
    outs = lambda c: [t.clone() for t in (c.h, c.gu, c.dx, c.dwg, c.dwu)]
    wants = [outs(c) for c in cases]
    block, one = cases[0].block, Case(M, K, F, "bf16", "silu", False)      # one handle, whatever the weights

    def passes(st):
        block.run(one.x, one.wg, one.wu, one.h, M, gu=one.gu, stream=st)
        block.grad(one.x, one.wg, one.wu, one.gu, one.dh, one.dx, one.dwg, one.dwu, M, stream=st)

    def take(c):
        for n in ("x", "wg", "wu", "dh"):
            getattr(one, n).copy_(getattr(c, n))

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        take(cases[1])
        passes(side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs(one), wants[1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        passes(torch.cuda.current_stream().cuda_stream)
    for c, want in zip(cases, wants):
        take(c)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs(one), want))


FORMS = {  # rows, K, F, product, block that is left out, what patdnn_gated_plan says
    "forward, one range": (2500, 700, 2600, 0, 13, dict(splits=1, blocks=11, few_rows=0)),
    "forward, split": (150, 20000, 256, 0, 2, dict(splits=35, few_rows=0)),
    "forward, rows of two tiles": (150, 4096, 256, 0, 2, dict(splits=8, few_rows=1, row_tiles=2)),
    "forward, few rows": (1, 4096, 8192, 0, 31, dict(splits=1, few_rows=1, blocks=64)),
    "forward, few rows, cluster of eight": (40, 4096, 256, 0, 2, dict(splits=8, few_rows=1)),
    "forward, few rows, more CTAs than SMs": (100, 200, 20000, 0, 3, dict(splits=1, few_rows=1)),
    "forward, several tiles": (5000, 130, 1000, 0, 7, dict(splits=1, grid=148)),
    "input, split": (40, 200, 2000, 1, 1, dict(splits=16)),
    "weights, split": (5000, 200, 200, 2, 4, dict(splits=16)),
}


@pytest.mark.parametrize("form", FORMS)
def test_a_wait_that_runs_out_is_reported_and_the_handle_keeps_working(form):
    """The bound is shortened to a few milliseconds and the copies of one block are left out, so that the consumers' wait for them runs out."""
    import torch
    from paper_2001_00138_b200 import binding as B
    M, K, F, product, skip, plan = FORMS[form]
    got = B.gated_plan(F, K, M, product)
    assert {k: got[k] for k in plan} == plan, got
    c = Case(M, K, F, "bf16", "silu", False)
    step = [lambda: c.forward(), lambda: c.backward(dw=False), lambda: c.backward(dx=False)][product]
    c.forward()
    step()
    want = [t.clone() for t in (c.h, c.dx, c.dwg, c.dwu)]
    c.block.debug_wait(1024, skip)
    with pytest.raises(B.PatdnnError) as e:
        step()
    assert e.value.status == E_DEVICE_TIMEOUT
    c.block.check()
    c.block.debug_wait(0, 0)
    if product == 0:
        c.h.fill_(float("nan"))
    step()
    assert all(torch.equal(a, b) or product != 0 and torch.isnan(b).all() for a, b in zip((c.h, c.dx, c.dwg, c.dwu), want))


def test_long_rows_of_x():
    """Rows so far apart that the last ones lie beyond 2^31 elements."""
    import torch
    from paper_2001_00138_b200 import binding as B
    M, K, F, ld = 40, 72, 64, 2 ** 31 // 39 + 64 - (2 ** 31 // 39) % 8
    g = torch.Generator(device="cuda").manual_seed(0)
    fx, fdx = (torch.zeros((M - 1) * ld + K, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x, dx = (torch.as_strided(t, (M, K), (ld, 1)) for t in (fx, fdx))
    x.copy_(torch.randint(-2, 3, (M, K), generator=g, device="cuda"))
    wg, wu = (torch.randint(-2, 3, (F, K), generator=g, device="cuda").bfloat16() for _ in range(2))
    h, gu, dh = (torch.randint(-2, 3, s, generator=g, device="cuda").bfloat16() for s in ((M, F), (M, 2, F), (M, F)))
    block = B.Gated(F, K, max_rows=M, act=B.ACT_NONE, x_row=ld, grad=True)
    block.run(x, wg, wu, h, M, stream=stream())
    block.grad(x, wg, wu, gu, dh, dx, None, None, M, stream=stream())
    block.check()
    same(h, ((x.double() @ wg.double().t()) * (x.double() @ wu.double().t())).bfloat16().double(), "h")
    same(dx, (dh.double() * gu[:, 1].double() @ wg.double() + dh.double() * gu[:, 0].double() @ wu.double()).bfloat16().double(), "dx")


def test_refusals_of_calls():
    import torch
    from paper_2001_00138_b200 import binding as B
    t = torch.zeros(64, 64, dtype=torch.float16, device="cuda")
    p = t.data_ptr()
    b = B.Gated(16, 24, max_rows=4, dtype=B.F16)
    refused(E_SHAPE, b.run, t, t, t, t, 5)
    refused(E_SHAPE, b.run, t, t, t, t, -1)
    refused(E_SCRATCH, b.grad, t, t, t, t, t, t, t, t, 1)
    b = B.Gated(16, 24, max_rows=4, dtype=B.F16, grad=True)
    for i in range(4):
        args = [t] * 4
        args[i] = 0
        refused(E_NULL, b.run, *args, 1)
        args[i] = p + (8 if i < 3 else 1)
        refused(E_SHAPE, b.run, *args, 1)
    refused(E_SHAPE, b.run, t, t, t, t, 1, gu=p + 1)
    for i in range(5):
        args = [t] * 8
        args[i] = 0
        refused(E_NULL, b.grad, *args, 1)
    refused(E_NULL, b.grad, t, t, t, t, t, t, None, t, 1)
    refused(E_NULL, b.grad, t, t, t, t, t, t, t, None, 1)
    for i in range(8):
        args = [t] * 8
        args[i] = p + 1
        refused(E_SHAPE, b.grad, *args, 1)
    odd = B.Gated(16, 24, max_rows=4, dtype=B.F16, x_row=25, w_row=27)     # such rows are packed, wherever they lie
    odd.run(p + 2, p + 4, p + 6, torch.zeros(4, 16, dtype=torch.float16, device="cuda"), 1, stream=stream())
    odd.check()


@pytest.mark.parametrize("name", ["relu", "silu"])
def test_gradient_where_the_gate_leaves_the_range_of_the_type(name):
    """g of +-2^17 is an infinity in half; the activation has its limits there: no gradient below, slope 1 above.  Exact values all the way."""
    import torch
    from paper_2001_00138_b200 import binding as B
    M, K, F = 40, 16, 72
    b = B.Gated(F, K, max_rows=M, dtype=B.F16, act=act_of(name), grad=True)
    x, dh = torch.zeros(M, K, device="cuda", dtype=torch.half), torch.zeros(M, F, device="cuda", dtype=torch.half)
    wg, wu = torch.zeros(F, K, device="cuda", dtype=torch.half), torch.zeros(F, K, device="cuda", dtype=torch.half)
    x[:, 0], x[:, 1] = 256.0, 1.0
    wg[0::2, 0], wg[1::2, 0] = 512.0, -512.0
    wu[:, 1] = 2.0 ** -8
    gu, h = torch.empty(M, 2, F, device="cuda", dtype=torch.half), torch.empty(M, F, device="cuda", dtype=torch.half)
    b.run(x, wg, wu, h, M, gu=gu, stream=stream())
    dh[:, 1::2] = 1.0                                      # below: nothing flows
    dh[:, 0::2] = 0.0
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    dh_below = dh.clone()
    torch.cuda.synchronize()
    assert torch.isinf(gu[:, 0]).all()
    assert torch.equal(h[:, 0::2], torch.full_like(h[:, 0::2], 512.0)) and not h[:, 1::2].any()
    g = gu.clone()
    g[:, 0, 0::2] = 1.0                                    # (the ones above apart: 0 * infinity has no value)
    b.grad(x, wg, wu, g, dh_below, dx, dwg, dwu, M, stream=stream())
    torch.cuda.synchronize()
    assert not dx.any() and not dwg.any() and not dwu.any()
    dh[:, 1::2] = 0.0
    dh[:, 0::2] = 1.0                                      # above: dg = dh u, du = dh g
    b.grad(x, wg, wu, gu, dh, dx, dwg, dwu, M, stream=stream())
    torch.cuda.synchronize()
    assert torch.equal(dwg[0::2, 1], torch.full_like(dwg[0::2, 1], M * 2.0 ** -8)) and torch.equal(dwg[0::2, 0], torch.full_like(dwg[0::2, 0], M * 1.0))
    assert torch.isinf(dwu[0::2, :2]).all() and not dwg[1::2].any()
    assert b.check() is None


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("M, K, F", [(1, 6899, 300), (5, 200, 72), (40, 77, 335), (128, 1000, 1333), (2, 64, 8), (1, 3, 9), (1, 5, 4), (3, 57, 17), (100, 120, 20), (17, 449, 1030)])
def test_weights_that_lie_anywhere(M, K, F, dtype):
    """Weights a row apart that is no whole number of 16-byte units, at bases that begin alike in a unit and that do not, between NaNs; and a row of
    either that is not finite, which spoils its own output alone."""
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = types(dtype)
    g = torch.Generator(device="cuda").manual_seed(M + K + F)

    def make(r, c):
        keep = torch.rand(r, c, generator=g, device="cuda") < min(1.0, 200.0 / K)
        return (torch.randint(-2, 3, (r, c), generator=g, device="cuda") * keep).to(tt)

    x, wg, wu = make(M, K), make(F, K), make(F, K)
    p, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    for wslack in (0, 1, 2, 3, 4, 7):
        if (K + wslack) % 8 == 0:
            continue
        b = B.Gated(F, K, max_rows=M + 3, dtype=dt, act=B.ACT_RELU, w_row=K + wslack, x_row=K + 3)
        for og, ou in ((0, 0), (1, 1), (5, 5), (7, 15), (2, 3), (0, 4)):
            (_, xs), (_, gs), (_, us) = spaced(x, 3, 1), spaced(wg, wslack, og), spaced(wu, wslack, ou)
            if (K + 3) % 8 == 0:
                xs = spaced(x, 3, 0)[1]
            fh, h = spaced(torch.zeros(M, F, dtype=tt), 0, 1)
            gu = torch.full((M, 2, F), float("nan"), dtype=tt, device="cuda")
            b.run(xs, gs, us, h, M, gu=gu, stream=stream())
            b.check()
            same(gu[:, 0], p, f"g {wslack} {og} {ou}")
            same(gu[:, 1], u, f"u {wslack} {og} {ou}")
            same(h, (p.clamp_min(0) * u).to(tt).double(), f"h {wslack} {og} {ou}")
            assert untouched(fh, h)
            one, two = F // 3, F // 2
            gs[one, K - 1] = float("inf")
            us[two, 0] = float("nan")
            gu.fill_(7)
            b.run(xs, gs, us, h, M, gu=gu, stream=stream())
            b.check()
            keep = torch.ones(F, dtype=torch.bool, device="cuda")
            keep[one], keep[two] = False, False
            same(h[:, keep], (p.clamp_min(0) * u).to(tt).double()[:, keep], f"h beside {wslack} {og} {ou}")
            assert torch.isnan(gu[:, 1, two]).all() and not torch.isfinite(gu[:, 0, one]).any()
        b.free()
