"""Group norm and linear layers at the ends of their ranges: many images, very many channels, one group or one per channel, long sums, and
the cluster splits of the product that the ordinary sizes do not reach.

References are fp64 on the device; bounds are those of test_gpu_norm and test_gpu_mx4.
"""
import pytest

import ops_ref as R
from test_gpu_linear_rows import held

pytestmark = pytest.mark.gpu
EPS = 1e-5


def mean_of(t, G):
    """Mean over the pixels and a group's channels of [N][P][C], per image and channel."""
    n, _, c = t.shape
    return t.reshape(n, -1, G, c // G).mean((1, 3)).repeat_interleave(c // G, 1)[:, None, :]


@pytest.mark.parametrize("N, P, C, G, dtype, act", [
    (65535, 2, 8, 2, "f32", "none"), (20000, 16, 32, 32, "f16", "silu"), (3000, 49, 64, 8, "bf16", "relu"),
    (1, 3, 2 ** 20, 1, "bf16", "silu"), (1, 3, 2 ** 20, 2 ** 20, "f32", "relu"), (2, 5, 2 ** 19, 1024, "f16", "silu"), (1, 40, 99991, 1, "f32", "none"),
    (3, 1000, 4098, 683, "f16", "relu")])
def test_group_norm_and_gradient(N, P, C, G, dtype, act):
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = {"f32": (torch.float32, B.F32), "f16": (torch.float16, B.F16), "bf16": (torch.bfloat16, B.BF16)}[dtype]
    st = torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device="cuda").manual_seed(C)
    x = (torch.randn(N, P, C, generator=g, device="cuda") * 1.5 + torch.randn(C, generator=g, device="cuda")).to(tt)
    dy = torch.randn(N, P, C, generator=g, device="cuda").to(tt)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g, device="cuda"), 0.3 * torch.randn(C, generator=g, device="cuda")
    h = B.GroupNorm(N, P, C, G, dtype=dt, act={"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU}[act], eps=EPS)
    y, dx, stats = torch.full_like(x, float("nan")), torch.full_like(x, float("nan")), torch.full((N, G, 2), float("nan"), device="cuda")
    h.run(x, gamma, beta, y, stats, st)
    v, d, ga, be = x.double(), dy.double(), gamma.double(), beta.double()
    mean = mean_of(v, G)
    rstd = (mean_of((v - mean) ** 2, G) + EPS) ** -0.5
    xh = (v - mean) * rstd
    z = xh * ga + be
    s = torch.sigmoid(z)
    ref = z if act == "none" else z.clamp_min(0) if act == "relu" else z * s
    size = ga.abs() * (xh.abs() + (mean * rstd).abs() + 1) + be.abs()
    torch.cuda.synchronize()
    assert ((y.double() - ref).abs() <= 1.1 * 34 * R.EPS24 * size + R.UNIT[dtype] * ref.abs() * 1.01 + R.TINY[dtype]).all()
    per = C // G
    exact = torch.stack([mean[:, 0, ::per], rstd[:, 0, ::per]], -1).float()
    dgamma, dbeta = (torch.full((C,), float("nan"), device="cuda") for _ in range(2))
    for _ in range(2):                                     # the second call finds the counters as the first left them
        h.grad(x, gamma, beta, exact, dy, dx, dgamma, dbeta, st)
    torch.cuda.synchronize()
    dz = d if act == "none" else torch.where(z > 0, d, torch.zeros_like(d)) if act == "relu" else d * s * (1 + z * (1 - s))
    u = dz * ga
    ref = rstd * (u - mean_of(u, G) - xh * mean_of(u * xh, G))
    size = rstd * (u.abs() + mean_of(u.abs(), G) + xh.abs() * mean_of((u * xh).abs(), G))
    zerr = 4 * R.EPS24 * ((xh.abs() + (mean * rstd).abs()) * ga.abs() + be.abs())
    sure = z.abs() > zerr if act == "relu" else torch.ones_like(z, dtype=torch.bool)
    assert sure.double().mean() > 0.99
    bound = 64 * R.EPS24 * size * (1 + (mean * rstd).abs()) + 0.6 * zerr * (d * ga).abs() * rstd + R.UNIT[dtype] * ref.abs() * 1.01 + R.TINY[dtype]
    assert (((dx.double() - ref).abs() <= bound) | ~sure).all()
    jump = torch.where(sure, torch.zeros_like(d), d.abs() * (1 + xh.abs())).sum((0, 1))
    # near its zero at z = -1.28 SiLU's slope is off by what z is off by and by the four roundings of the sigmoid, however small dz is there
    slope = (0.6 * zerr + 4 * R.EPS24) * (d * xh).abs() if act == "silu" else torch.zeros_like(d)
    bound = 64 * R.EPS24 * (dz.abs() * (xh.abs() + (mean * rstd).abs())) + slope
    assert ((dgamma.double() - (dz * xh).sum((0, 1))).abs() <= bound.sum((0, 1)) + jump).all()
    assert ((dbeta.double() - dz.sum((0, 1))).abs() <= 64 * R.EPS24 * dz.abs().sum((0, 1)) + (0.6 * zerr * d.abs()).sum((0, 1)) + jump).all()


@pytest.mark.parametrize("N, P, C, G", [(20000, 16, 40, 4), (1, 3, 2 ** 20, 16), (2, 1000, 4098, 683)])
def test_group_norm_into_4_bit_rows(N, P, C, G):
    import torch
    from paper_2001_00138_b200 import binding as B
    st = torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device="cuda").manual_seed(C)
    x = (torch.randn(N, P, C, generator=g, device="cuda") * 1.5 + torch.randn(C, generator=g, device="cuda")).bfloat16()
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g, device="cuda"), 0.3 * torch.randn(C, generator=g, device="cuda")
    h = B.GroupNorm(N, P, C, G, dtype=B.BF16, act=B.ACT_RELU, eps=EPS)
    mx, stats = torch.full((B.mx4_bytes(N * P, C),), 255, dtype=torch.uint8, device="cuda"), torch.full((N, G, 2), float("nan"), device="cuda")
    h.run_mx4(x, gamma, beta, mx, stats, st)
    out, twice = torch.empty(N * P, C, device="cuda"), torch.empty(N * P, C, device="cuda")
    B.mx4_dequantize(mx, out, N * P, C, stream=st)
    mean, rstd = (stats[..., k].repeat_interleave(C // G, 1)[:, None, :] for k in (0, 1))
    z = ((x.float() - mean) * rstd * gamma + beta).clamp_min(0).reshape(N * P, C)
    again = torch.full_like(mx, 255)
    B.mx4_quantize(z, again, N * P, C, stream=st)
    B.mx4_dequantize(again, twice, N * P, C, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(out, twice)                          # the steps rounded one by one, then the quantisation that test_gpu_mx4 checks


@pytest.mark.parametrize("rows, K, F, plan", [
    (128, 8192, 300, dict(splits=8, tile_rows=128)), (100, 16384, 100, dict(splits=8, tile_rows=112)), (300, 4100, 200, dict(splits=4, tile_rows=128)),
    (65, 6000, 1000, dict(splits=4, tile_rows=80)), (40, 2300, 77, dict(splits=8, tile_rows=48, column_tiles=9)),
    (5, 2 ** 20, 40, dict(splits=8, quantises=1)), (200, 2 ** 20, 100, dict(splits=8)), (2, 40, 2 ** 20, dict(splits=1, quantises=1)), (20, 40, 2 ** 20, dict(persistent=0))])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_linear(rows, K, F, plan, dtype):
    import torch
    from paper_2001_00138_b200 import binding as B
    got = B.linear_plan(F, K, rows)
    assert {k: got[k] for k in plan} == plan, got
    tt, dt = {"f32": (torch.float32, B.F32), "f16": (torch.float16, B.F16), "bf16": (torch.bfloat16, B.BF16)}[dtype]
    st = torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device="cuda").manual_seed(K + F)
    x, w, b = held(rows, K, g), held(F, K, g) / 8, torch.randn(F, generator=g, device="cuda")
    lin = B.Linear(w.to(tt), F, K, max_rows=rows, dtype=dt, bias=b, stream=st)
    y = torch.full((rows, F), float("nan"), dtype=tt, device="cuda")
    lin.run(x.to(tt), y, rows, stream=st)
    lin.check()
    ref = x.double() @ w.double().t() + b.double()
    size = x.double().abs() @ w.double().abs().t() + b.double().abs()
    bound = 1.1 * (K / 64 + 10) * 2.0 ** -23 * size + R.UNIT[dtype] * ref.abs() * 1.01 + R.TINY[dtype]
    assert ((y.double() - ref).abs() <= bound).all()
