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
