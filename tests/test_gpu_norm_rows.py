"""Group norm written straight into 4-bit rows: the values are formed step by step in fp32, each step rounded, before they are quantised.

4-bit rounding jumps, so the steps are part of the definition: fl(fl(fl(x - mean) * rstd) * gamma) + beta, with the statistics that the call
returns.  beta is chosen so that in every channel one pixel lands exactly on a middle between two codes when the steps are rounded as
stated; a fused multiply-add would leave it beside the middle in about one channel of four.
"""
import numpy as np
import pytest

import ops_ref as R

pytestmark = pytest.mark.gpu
F = np.float32


def run(h, B, x, gamma, beta, rows, C, G, N):
    import torch
    st = torch.cuda.current_stream().cuda_stream
    mx = torch.full((B.mx4_bytes(rows, C),), 255, dtype=torch.uint8, device="cuda")
    stats, out = torch.empty(N, G, 2, device="cuda"), torch.empty(rows, C, device="cuda")
    h.run_mx4(x, torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda(), mx, stats, st)
    B.mx4_dequantize(mx, out, rows, C, stream=st)
    torch.cuda.synchronize()
    return stats.cpu().numpy(), out.cpu().numpy()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N, P, C, G, act, slack", [
    (1, 64, 512, 16, "none", 0), (2, 300, 256, 32, "relu", 0), (3, 77, 96, 8, "none", 8), (2, 50, 320, 32, "relu", 3), (1, 9, 1000, 125, "none", 0),
    (1, 60000, 64, 1, "none", 0), (2, 70001, 36, 4, "relu", 0)])
def test_the_steps_are_rounded_one_by_one(N, P, C, G, act, slack, dtype):
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = {"f32": (torch.float32, B.F32), "f16": (torch.float16, B.F16), "bf16": (torch.bfloat16, B.BF16)}[dtype]
    rng = np.random.default_rng(P)
    x = torch.from_numpy(np.clip(rng.standard_normal((N, P, C)), -3, 3)).to(tt)
    wide = torch.zeros(N, P, C + slack, dtype=tt, device="cuda")
    wide[..., :C] = x
    xs = x.float().numpy()
    gamma = (1 + 0.1 * rng.standard_normal(C)).astype(F)
    gamma[::32] = 0
    h = B.GroupNorm(N, P, C, G, dtype=dt, act={"none": B.ACT_NONE, "relu": B.ACT_RELU}[act], x_pixel=C + slack)
    rows = N * P
    stats, _ = run(h, B, wide, gamma, np.zeros(C, F), rows, C, G, N)
    mean, rstd = (np.repeat(stats[..., k], C // G, axis=1)[:, None, :] for k in (0, 1))
    with np.errstate(all="raise", under="ignore"):
        p = ((xs - mean).astype(F) * rstd).astype(F) * gamma
    assert p.dtype == F
    beta = np.zeros(C, F)
    for c in range(C):
        at = p[0, :2000, c]
        fits = [at[(at >= 2.0 ** np.ceil(np.log2(k))) & (at <= 2 * k)] for k in (0.75, 1.75, 3.5)]
        found = [(k, v[0]) for k, v in zip((0.75, 1.75, 3.5), fits) if v.size]
        if found:
            k, v = found[c % len(found)]
            beta[c] = F(k) - v                                     # exact: v is within [k, 2k]
    beta[::32] = 6                                                 # every block's largest magnitude lies in [4, 8): scale 1
    again, got = run(h, B, wide, gamma, beta, rows, C, G, N)
    assert np.array_equal(stats, again)
    z = (p + beta).astype(F)
    want = R.quantise(R.act(z.reshape(rows, C).astype(np.float64), act))
    off = got != want
    assert not off.any(), f"{int(off.sum())} of {off.size} values are not the stated ones, first at {np.argwhere(off)[:4].tolist()}"


@pytest.mark.parametrize("N, P, C, G, dtype", [(32, 3136, 64, 32, "bf16"), (64, 196, 512, 32, "f32"), (8, 60000, 64, 32, "bf16"), (16, 20011, 48, 16, "f32")])
def test_statistics_are_rounded_about_once(N, P, C, G, dtype):
    """mean and rstd equal fl(mean) and rsqrt(fl(fl(variance) + eps)) in at least 7 groups of 8, and are a step of fp32 away in the others.

    A thread's own fp32 sums are off by a few 2^-25 of the values' spread s; over the threads of a group that leaves some 2^-25 s / 8, joined
    without further rounding.  With means of about 2 s, whose steps are 2^-22 s, and variances whose steps are 2^-23 of them, the rounding then
    differs in about one group of 20."""
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = {"f32": (torch.float32, B.F32), "bf16": (torch.bfloat16, B.BF16)}[dtype]
    g = torch.Generator(device="cuda").manual_seed(P)
    x = (torch.randn(N, P, C, generator=g, device="cuda") + 2.5).to(tt)
    one, zero = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    var, mean = torch.var_mean(x.double().reshape(N, P, G, -1), dim=(1, 3), correction=0)
    rstd = torch.rsqrt(var.float() + 1e-5)
    h = B.GroupNorm(N, P, C, G, dtype=dt)
    y, mx = torch.empty_like(x), torch.empty(B.mx4_bytes(N * P, C), dtype=torch.uint8, device="cuda")
    for call in (lambda s: h.run(x, one, zero, y, s, st), lambda s: h.run_mx4(x, one, zero, mx, s, st)):
        stats = torch.empty(N, G, 2, device="cuda")
        call(stats)
        torch.cuda.synchronize()
        for got, want, what in ((stats[..., 0], mean.float(), "mean"), (stats[..., 1], rstd, "rstd")):
            step = (got.view(torch.int32) if got.is_contiguous() else got.contiguous().view(torch.int32)) - want.contiguous().view(torch.int32)
            assert step.abs().max() <= 1, (what, int(step.abs().max()))
            assert (step != 0).float().mean() <= 1 / 8, (what, (step != 0).float().mean().item())
