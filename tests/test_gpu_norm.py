"""Group norm with an activation (channels last) and its gradient against 64-bit statements.

Bounds, fixed before the first run.  fp32 sums are trees and short runs of at most a few dozen terms, so the mean is off by at most 32
roundings of the largest magnitude in it, and likewise rstd relative to itself; an output then is off by 32 roundings of
|gamma| (|xh| + |mean| rstd + 1) + |beta|, plus its own rounding to the storage type.  The fast exponential of SiLU is good to
2 + 1.2 |z| ulp, which adds at most two more roundings of |z|; both activations have slopes below 1.1.
"""
import numpy as np
import pytest

import ops_ref as R

pytestmark = pytest.mark.gpu
EPS = 1e-5


def setup(N, P, C, G, dtype, act, *, xs=0, ys=0, gap=0, seed=0, mean=1.0):
    """Inputs in the storage type (and the same as float64), and a handle; xs, ys: elements between pixels, gap: between images."""
    import torch
    from paper_2001_00138_b200 import binding as B
    tt = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(N, P, C, generator=g) * (0.5 + torch.rand(C, generator=g)) + mean * torch.randn(C, generator=g)).to(tt)
    dy = torch.randn(N, P, C, generator=g).to(tt)
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g), 0.3 * torch.randn(C, generator=g)

    def place(v, slack):
        row = P * (C + slack) + gap
        flat = torch.full((N * row + 16,), float("nan"), dtype=tt, device="cuda")
        view = torch.as_strided(flat, (N, P, C), (row, C + slack, 1))
        view.copy_(v)
        return flat, view

    h = B.GroupNorm(N, P, C, G, dtype={"f32": B.F32, "f16": B.F16, "bf16": B.BF16}[dtype],
                    act={"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU}[act], eps=EPS,
                    x_pixel=C + xs, x_image=P * (C + xs) + gap, y_pixel=C + ys, y_image=P * (C + ys) + gap)
    fx, vx = place(x, xs)
    fd, vd = place(dy, ys)
    return dict(h=h, x=vx, dy=vd, gamma=gamma.cuda(), beta=beta.cuda(), x64=x.double().numpy(), dy64=dy.double().numpy(),
                g64=gamma.double().numpy(), b64=beta.double().numpy(), place=place, tt=tt, keep=(fx, fd), st=torch.cuda.current_stream().cuda_stream)


def forward(s, N, P, C, G, dtype, act, ys=0, what=""):
    import torch
    flat, y = s["place"](torch.full((N, P, C), 7.0), ys)
    stats = torch.full((N, G, 2), float("nan"), device="cuda")
    s["h"].run(s["x"], s["gamma"], s["beta"], y, stats, s["st"])
    torch.cuda.synchronize()
    ref = R.norm(s["x64"], s["g64"], s["b64"], G, EPS, act)
    size = np.abs(s["g64"]) * (np.abs(ref["xh"]) + np.abs(ref["mc"]) * ref["rc"] + 1) + np.abs(s["b64"])
    R.within(y.double().cpu().numpy(), ref["y"], 1.1 * 34 * R.EPS24 * size + R.UNIT[dtype] * np.abs(ref["y"]) * 1.01 + R.TINY[dtype], "y " + what)
    top = np.abs(s["x64"]).max()
    st = stats.double().cpu().numpy()
    R.within(st[..., 0], ref["mean"], 32 * R.EPS24 * top, "mean " + what)
    R.within(st[..., 1], ref["rstd"], 32 * R.EPS24 * ref["rstd"] * (1 + np.abs(ref["mean"]) * ref["rstd"]), "rstd " + what)
    # nothing outside the tensor was written
    inside = torch.zeros_like(flat, dtype=torch.bool)
    torch.as_strided(inside, y.shape, y.stride()).fill_(True)
    assert torch.isnan(flat[~inside]).all(), what
    return stats


SHAPES = [  # N, P, C, G
    (1, 1, 1, 1), (1, 1, 32, 32), (2, 1, 64, 8), (1, 49, 512, 32), (3, 7, 10, 5), (2, 50, 6, 1), (2, 837, 320, 32), (1, 3, 96, 3),
    (5, 100, 24, 4), (2, 33, 2048, 16), (1, 17, 4099, 1), (2, 4096, 64, 32), (1, 70000, 8, 2), (1, 9, 1000, 125), (4, 31, 33, 11),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype):
    N, P, C, G = shape
    act = ["none", "relu", "silu"][(N + P + C) % 3]
    s = setup(N, P, C, G, dtype, act, seed=P)
    forward(s, N, P, C, G, dtype, act, what=f"{shape} {dtype} {act}")


@pytest.mark.parametrize("dtype, xs, ys, gap", [("f32", 4, 0, 0), ("f32", 1, 3, 5), ("f16", 8, 16, 8), ("bf16", 2, 0, 2), ("bf16", 0, 1, 0), ("f16", 0, 0, 1)])
@pytest.mark.parametrize("shape", [(3, 61, 48, 6), (2, 20000, 16, 4)])
def test_forward_strides(shape, dtype, xs, ys, gap):
    N, P, C, G = shape
    s = setup(N, P, C, G, dtype, "silu", xs=xs, ys=ys, gap=gap, seed=3)
    forward(s, N, P, C, G, dtype, "silu", ys=ys, what=f"{shape} {dtype} {xs} {ys} {gap}")


@pytest.mark.parametrize("shape", [(2, 400, 32, 8), (1, 300000, 32, 8)])
def test_a_large_mean_does_not_eat_the_variance(shape):
    N, P, C, G = shape
    s = setup(N, P, C, G, "f32", "none", seed=5, mean=3000.0)
    forward(s, N, P, C, G, "f32", "none", what="large mean")


@pytest.mark.parametrize("shape", [(3, 60, 64, 8), (3, 40000, 64, 8)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_not_finite_stays_in_its_image_and_group(shape, bad):
    import torch
    N, P, C, G = shape
    s = setup(N, P, C, G, "f32", "relu", seed=6)
    y0, y1 = (torch.empty(N, P, C, device="cuda") for _ in range(2))
    s["h"].run(s["x"], s["gamma"], s["beta"], y0, None, s["st"])
    s["x"][1, P // 2, 17] = bad                            # image 1, group 2
    s["h"].run(s["x"], s["gamma"], s["beta"], y1, None, s["st"])
    torch.cuda.synchronize()
    hit = torch.zeros(N, P, C, dtype=torch.bool, device="cuda")
    hit[1, :, 16:24] = True
    assert torch.isnan(y1[hit]).all()
    assert torch.equal(y1[~hit], y0[~hit])


def backward(s, N, P, C, G, dtype, act, xs=0, what=""):
    import torch
    ref = R.norm_grad(s["x64"], s["g64"], s["b64"], G, EPS, act, s["dy64"])
    stats = torch.from_numpy(np.stack([ref["fwd"]["mean"], ref["fwd"]["rstd"]], -1)).float().cuda()
    flat, dx = s["place"](torch.full((N, P, C), 7.0), xs)
    dgamma, dbeta = (torch.full((C,), float("nan"), device="cuda") for _ in range(2))
    s["h"].grad(s["x"], s["gamma"], s["beta"], stats, s["dy"], dx, dgamma, dbeta, s["st"])
    torch.cuda.synchronize()
    f = ref["fwd"]
    # xh carries the rounding of mean and rstd (2 roundings of |mean| rstd and of |xh|); the slope of SiLU changes by at most half of
    # what z does, ReLU's jumps at 0: elements whose z is nearer to 0 than its error are left out (there are none to speak of)
    wobble = 4 * R.EPS24 * (np.abs(f["xh"]) + np.abs(f["mc"]) * f["rc"])
    zerr = wobble * np.abs(s["g64"]) + 4 * R.EPS24 * np.abs(s["b64"])
    sure = np.abs(f["z"]) > zerr if act == "relu" else np.ones_like(f["z"], bool)
    assert sure.mean() > 0.99
    extra = 0.6 * zerr * np.abs(s["dy64"] * s["g64"]) * f["rc"]
    bound = 64 * R.EPS24 * (ref["dx_size"] * (1 + np.abs(f["mc"]) * f["rc"])) + extra + R.UNIT[dtype] * np.abs(ref["dx"]) * 1.01 + R.TINY[dtype]
    R.within(np.where(sure, dx.double().cpu().numpy(), ref["dx"]), ref["dx"], bound, "dx " + what)
    # sums of N * P terms in runs per thread, then a tree: 64 roundings of the sum of magnitudes (jumps of ReLU's slope: see above)
    jump = np.where(sure, 0, np.abs(s["dy64"]) * (1 + np.abs(f["xh"]))).sum((0, 1))
    R.within(dgamma.double().cpu().numpy(), ref["dgamma"], 64 * R.EPS24 * ref["dgamma_size"] + jump, "dgamma " + what)
    R.within(dbeta.double().cpu().numpy(), ref["dbeta"], 64 * R.EPS24 * ref["dbeta_size"] + (0.6 * zerr * np.abs(s["dy64"])).sum((0, 1)) + jump, "dbeta " + what)
    inside = torch.zeros_like(flat, dtype=torch.bool)
    torch.as_strided(inside, dx.shape, dx.stride()).fill_(True)
    assert torch.isnan(flat[~inside]).all(), what
    return dx, dgamma, dbeta


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradient(shape, dtype):
    N, P, C, G = shape
    act = ["none", "relu", "silu"][(N + P + C + 1) % 3]
    s = setup(N, P, C, G, dtype, act, seed=P + 1)
    backward(s, N, P, C, G, dtype, act, what=f"{shape} {dtype} {act}")


@pytest.mark.parametrize("dtype, xs, ys, gap", [("f32", 4, 0, 0), ("f32", 1, 3, 5), ("f16", 8, 16, 8), ("bf16", 2, 0, 2), ("bf16", 0, 1, 0)])
@pytest.mark.parametrize("shape", [(3, 61, 48, 6), (2, 20000, 16, 4)])
def test_gradient_strides(shape, dtype, xs, ys, gap):
    N, P, C, G = shape
    s = setup(N, P, C, G, dtype, "silu", xs=xs, ys=ys, gap=gap, seed=3)
    backward(s, N, P, C, G, dtype, "silu", xs=xs, what=f"{shape} {dtype} {xs} {ys} {gap}")


@pytest.mark.parametrize("act", ["none", "silu"])
def test_gradient_against_differences(act):
    """(L(x + h v) - L(x - h v)) / 2h = <dL/dx, v> for L = sum(y * dy), and the same for gamma and beta, through the forward kernel.
    With h = 2^-5 the third-order term is below h^2 of the first (all values are of order 1) and fp32 rounding of the outputs adds
    2^-24 * sqrt(count) / h: 0.5 % of |dL| |v| / sqrt(count) per direction, checked at 2 % of it."""
    import torch
    N, P, C, G = 2, 40, 48, 6
    s = setup(N, P, C, G, "f32", act, seed=9)
    stats = torch.empty(N, G, 2, device="cuda")
    y = torch.empty(N, P, C, device="cuda")
    s["h"].run(s["x"], s["gamma"], s["beta"], y, stats, s["st"])
    dx, dgamma, dbeta = torch.empty(N, P, C, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    s["h"].grad(s["x"], s["gamma"], s["beta"], stats, s["dy"], dx, dgamma, dbeta, s["st"])

    def loss(x, gamma, beta):
        s["h"].run(x.contiguous(), gamma, beta, y, None, s["st"])
        return (y.double() * s["dy"].double()).sum().item()

    h = 2.0 ** -5
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        v, vg, vb = torch.randn(N, P, C, generator=g).cuda(), torch.randn(C, generator=g).cuda(), torch.randn(C, generator=g).cuda()
        x, ga, be = s["x"].contiguous(), s["gamma"], s["beta"]
        for got, grad, d in ((loss(x + h * v, ga, be) - loss(x - h * v, ga, be), dx, v), (loss(x, ga + h * vg, be) - loss(x, ga - h * vg, be), dgamma, vg),
                             (loss(x, ga, be + h * vb) - loss(x, ga, be - h * vb), dbeta, vb)):
            want = (grad.double() * d.double()).sum().item()
            assert abs(got / (2 * h) - want) <= 0.02 * (grad.norm() * d.norm()).item(), (act, seed)


def test_gradient_of_an_empty_batch_is_zero():
    import torch
    from paper_2001_00138_b200 import binding as B
    h = B.GroupNorm(0, 5, 16, 4)
    dgamma, dbeta = torch.ones(16, device="cuda"), torch.ones(16, device="cuda")
    h.grad(0, 0, 0, 0, 0, 0, dgamma, dbeta, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert not dgamma.any() and not dbeta.any()


@pytest.mark.parametrize("shape", [(4, 300, 64, 16), (2, 50000, 32, 4)])
def test_the_same_call_gives_the_same_bits(shape):
    N, P, C, G = shape
    import torch
    s = setup(N, P, C, G, "bf16", "silu", seed=11)
    a = backward(s, N, P, C, G, "bf16", "silu")
    for _ in range(5):
        b = backward(s, N, P, C, G, "bf16", "silu")
        assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_another_stream():
    import torch
    N, P, C, G = 4, 900, 64, 16
    s = setup(N, P, C, G, "f32", "silu", seed=12)
    side = torch.cuda.Stream()
    x2 = torch.zeros_like(s["x"], memory_format=torch.contiguous_format)
    y = torch.empty(N, P, C, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)                       # the copy below is late: a kernel on the wrong stream would read zeros
        x2.copy_(s["x"])
        s["h"].run(x2, s["gamma"], s["beta"], y, None, side.cuda_stream)
    side.synchronize()
    ref = R.norm(s["x64"], s["g64"], s["b64"], G, EPS, "silu")["y"]
    assert np.abs(y.double().cpu().numpy() - ref).max() < 1e-4


def test_null_pointers_are_refused():
    from paper_2001_00138_b200 import binding as B
    h = B.GroupNorm(1, 4, 8, 2)
    for call in (lambda: h.run(0, 64, 64, 64), lambda: h.run(64, 64, 64, 0), lambda: h.run_mx4(64, 64, 64, 0), lambda: h.grad(64, 64, 64, 0, 64, 64, 64, 64)):
        with pytest.raises(B.PatdnnError) as e:
            call()
        assert e.value.status == 1
    for call in (lambda: h.run_mx4(64, 64, 64, 72), lambda: h.run(66, 64, 64, 64), lambda: h.run(64, 64, 64, 64, stats=68), lambda: h.run(64, 66, 64, 64),
                 lambda: h.grad(64, 64, 64, 64, 64, 66, 64, 64), lambda: h.grad(64, 64, 64, 68, 64, 64, 64, 64)):
        with pytest.raises(B.PatdnnError) as e:
            call()
        assert e.value.status == 2


@pytest.mark.parametrize("P", [40, 60000])
def test_offsets_beyond_32_bits(P):
    """The second image begins 2^31 + 8 elements behind the first, in x, y, dy and dx."""
    import torch
    from paper_2001_00138_b200 import binding as B
    N, C, G = 2, 64, 8
    far = 2 ** 31 + 8
    g = torch.Generator().manual_seed(P)
    x = (torch.randn(N, P, C, generator=g) + torch.randn(C, generator=g)).bfloat16()
    dy = torch.randn(N, P, C, generator=g).bfloat16()
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=g), 0.3 * torch.randn(C, generator=g)

    def place(v):
        flat = torch.empty(far + P * C, dtype=torch.bfloat16, device="cuda")
        view = torch.as_strided(flat, (N, P, C), (far, C, 1))
        view.copy_(v)
        return view

    xv, dv, y, dx = place(x), place(dy), place(torch.zeros(N, P, C)), place(torch.zeros(N, P, C))
    h = B.GroupNorm(N, P, C, G, dtype=B.BF16, act=B.ACT_SILU, eps=EPS, x_image=far, y_image=far)
    stats = torch.empty(N, G, 2, device="cuda")
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    h.run(xv, gamma.cuda(), beta.cuda(), y, stats, st)
    h.grad(xv, gamma.cuda(), beta.cuda(), stats, dv, dx, dgamma, dbeta, st)
    torch.cuda.synchronize()
    ref = R.norm_grad(x.double().numpy(), gamma.double().numpy(), beta.double().numpy(), G, EPS, "silu", dy.double().numpy())
    f = ref["fwd"]
    size = np.abs(gamma.double().numpy()) * (np.abs(f["xh"]) + np.abs(f["mc"]) * f["rc"] + 1) + np.abs(beta.double().numpy())
    R.within(y.double().cpu().numpy(), f["y"], 40 * R.EPS24 * size + R.UNIT["bf16"] * np.abs(f["y"]) * 1.01 + R.TINY["bf16"], "y")
    R.within(dx.double().cpu().numpy(), ref["dx"], 128 * R.EPS24 * ref["dx_size"] * (1 + np.abs(f["mc"]) * f["rc"]) + R.UNIT["bf16"] * np.abs(ref["dx"]) * 1.01 + 1e-6, "dx")
    R.within(dbeta.double().cpu().numpy(), ref["dbeta"], 128 * R.EPS24 * ref["dbeta_size"], "dbeta")
