"""Group norm over tensors that the two-pass form takes in several runs of images: five images in runs of two, two and one (or three and two),
whose pixels are not a multiple of the 128 rows of a tile, so that row tiles of the 4-bit form belong to two launches.

Bounds are those of test_gpu_norm, evaluated in fp64 on the device.
"""
import pytest

import ops_ref as R

pytestmark = pytest.mark.gpu
EPS = 1e-5
N, C, G = 5, 64, 16


def inputs(P, dtype, slack=0):
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = {"f32": (torch.float32, B.F32), "f16": (torch.float16, B.F16), "bf16": (torch.bfloat16, B.BF16)}[dtype]
    g = torch.Generator(device="cuda").manual_seed(P)
    wide = torch.zeros(N, P, C + slack, dtype=tt, device="cuda")
    x = wide[..., :C]
    spread, mean = 0.5 + torch.rand(C, generator=g, device="cuda"), torch.randn(N, 1, C, generator=g, device="cuda")
    for n in range(N):                                     # every image has its own statistics
        x[n] = (torch.randn(P, C, generator=g, device="cuda") * spread * (n + 1) + mean[n]).to(tt)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g, device="cuda"), 0.3 * torch.randn(C, generator=g, device="cuda")
    return tt, dt, g, x, gamma, beta, torch.cuda.current_stream().cuda_stream


def groups(t):
    """Mean over an image's pixels and a group's channels of [P][C], per channel."""
    return t.reshape(t.shape[0], G, -1).mean((0, 2)).repeat_interleave(C // G)


def runs(call):
    """The runs of a call: three launches each."""
    from paper_2001_00138_b200 import binding as B
    before = B.launch_count()
    call()
    return (B.launch_count() - before) / 3


@pytest.mark.parametrize("P, dtype, slack, many", [(468751, "bf16", 0, 3), (410001, "f16", 8, 2), (234377, "f32", 0, 3), (440003, "bf16", 3, 3)])
def test_forward(P, dtype, slack, many):
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt, g, x, gamma, beta, st = inputs(P, dtype, slack)
    h = B.GroupNorm(N, P, C, G, dtype=dt, act=B.ACT_SILU, eps=EPS, x_pixel=C + slack)
    y, stats = torch.full((N, P, C), float("nan"), dtype=tt, device="cuda"), torch.full((N, G, 2), float("nan"), device="cuda")
    assert runs(lambda: h.run(x, gamma, beta, y, stats, st)) == many
    torch.cuda.synchronize()
    for n in range(N):
        v = x[n].double()
        mean = groups(v)
        rstd = (groups((v - mean) ** 2) + EPS) ** -0.5
        xh = (v - mean) * rstd
        z = xh * gamma.double() + beta.double()
        ref = z / (1 + torch.exp(-z))
        size = gamma.double().abs() * (xh.abs() + (mean * rstd).abs() + 1) + beta.double().abs()
        bound = 1.1 * 34 * R.EPS24 * size + R.UNIT[dtype] * ref.abs() * 1.01 + R.TINY[dtype]
        assert ((y[n].double() - ref).abs() <= bound).all(), n
        per = C // G
        assert ((stats[n, :, 0].double() - mean[::per]).abs() <= 32 * R.EPS24 * v.abs().max()).all(), n
        assert ((stats[n, :, 1].double() / rstd[::per] - 1).abs() <= 32 * R.EPS24 * (1 + (mean * rstd)[::per].abs())).all(), n


@pytest.mark.parametrize("P, dtype, slack, many", [(468751, "bf16", 0, 3), (410001, "f16", 8, 2), (234377, "f32", 0, 3), (440003, "bf16", 3, 3)])
def test_4_bit_rows(P, dtype, slack, many):
    """Equal, code for code, to the steps rounded one by one with the statistics that the call returns."""
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt, g, x, gamma, beta, st = inputs(P, dtype, slack)
    h = B.GroupNorm(N, P, C, G, dtype=dt, act=B.ACT_RELU, eps=EPS, x_pixel=C + slack)
    mx, stats = torch.full((B.mx4_bytes(N * P, C),), 255, dtype=torch.uint8, device="cuda"), torch.full((N, G, 2), float("nan"), device="cuda")
    assert runs(lambda: h.run_mx4(x, gamma, beta, mx, stats, st)) == many
    out = torch.empty(N * P, C, device="cuda")
    B.mx4_dequantize(mx, out, N * P, C, stream=st)
    torch.cuda.synchronize()
    for n in range(N):
        mean, rstd = (stats[n, :, k].repeat_interleave(C // G) for k in (0, 1))
        v = x[n].double()
        true = (groups((v - groups(v)) ** 2) + EPS) ** -0.5
        assert ((rstd.double() / true - 1).abs() <= 32 * R.EPS24 * (1 + (groups(v) * true).abs())).all(), n
        z = ((x[n].float() - mean) * rstd * gamma + beta).clamp_min(0).double().reshape(P, -1, 32)
        top = z.amax(-1, keepdim=True)
        scale = torch.where(top > 0, torch.ldexp(torch.ones_like(top), torch.frexp(top)[1] - 3), torch.ones_like(top))
        r = z / scale
        step = torch.where(r < 2, 0.5, torch.where(r < 4, 1.0, 2.0)).double()
        want = ((torch.round(r / step) * step).clamp_max(6) * scale).reshape(P, C)
        got = out[n * P:(n + 1) * P].double()
        assert torch.equal(got, want), (n, (got != want).nonzero()[:4].tolist())


@pytest.mark.parametrize("P, dtype, act", [(300001, "bf16", "silu"), (150001, "f32", "none"), (280003, "f16", "silu")])
def test_gradient(P, dtype, act):
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt, g, x, gamma, beta, st = inputs(P, dtype)
    dy = torch.empty_like(x)
    for n in range(N):
        dy[n] = torch.randn(P, C, generator=g, device="cuda").to(tt)
    ga, be = gamma.double(), beta.double()
    stats, per = torch.empty(N, G, 2, device="cuda"), C // G
    for n in range(N):
        v = x[n].double()
        m = groups(v)
        stats[n, :, 0], stats[n, :, 1] = m[::per].float(), ((groups((v - m) ** 2) + EPS) ** -0.5)[::per].float()
    h = B.GroupNorm(N, P, C, G, dtype=dt, act=B.ACT_SILU if act == "silu" else B.ACT_NONE, eps=EPS)
    dx = torch.full_like(x, float("nan"))
    dgamma, dbeta = (torch.full((C,), float("nan"), device="cuda") for _ in range(2))
    assert runs(lambda: h.grad(x, gamma, beta, stats, dy, dx, dgamma, dbeta, st)) == 3
    torch.cuda.synchronize()
    total = {k: torch.zeros(C, dtype=torch.float64, device="cuda") for k in ("dgamma", "dbeta", "gamma_size", "beta_size", "slack")}
    for n in range(N):
        v, d = x[n].double(), dy[n].double()
        mean = groups(v)
        rstd = (groups((v - mean) ** 2) + EPS) ** -0.5
        xh = (v - mean) * rstd
        z = xh * ga + be
        s = torch.sigmoid(z)
        dz = d * s * (1 + z * (1 - s)) if act == "silu" else d
        u = dz * ga
        ref = rstd * (u - groups(u) - xh * groups(u * xh))
        size = rstd * (u.abs() + groups(u.abs()) + xh.abs() * groups((u * xh).abs()))
        zerr = 4 * R.EPS24 * ((xh.abs() + (mean * rstd).abs()) * ga.abs() + be.abs())
        bound = 64 * R.EPS24 * size * (1 + (mean * rstd).abs()) + 0.6 * zerr * (d * ga).abs() * rstd + R.UNIT[dtype] * ref.abs() * 1.01 + R.TINY[dtype]
        assert ((dx[n].double() - ref).abs() <= bound).all(), n
        total["dgamma"] += (dz * xh).sum(0)
        total["dbeta"] += dz.sum(0)
        total["gamma_size"] += (dz.abs() * (xh.abs() + (mean * rstd).abs())).sum(0)
        total["beta_size"] += dz.abs().sum(0)
        total["slack"] += (0.6 * zerr * d.abs()).sum(0)
    assert ((dgamma.double() - total["dgamma"]).abs() <= 64 * R.EPS24 * total["gamma_size"]).all()
    assert ((dbeta.double() - total["dbeta"]).abs() <= 64 * R.EPS24 * total["beta_size"] + total["slack"]).all()
