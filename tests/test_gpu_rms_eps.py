"""RMS norm with an eps anywhere in fp32's range.  Bounds as in test_gpu_rms."""
import pytest

import ff_ref as R
from ff_ref import stream
from test_gpu_rms import adds, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-30, 0.9e-18, 1.1e-18, 1.0, 1e30, 0.9e38, 1.1e38, 2.5e38, 3.4e38])
@pytest.mark.parametrize("C", [7, 60, 1000, 9000])
def test_any_eps(C, eps):
    import torch
    from paper_2001_00138_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(C)
    magnitude = torch.tensor([1e-30, 1e-18, 1e-9, 1.0, 1e9, 1e15, 1e18, 1e19, 1e30], device="cuda")[:, None]
    x = torch.randn(9, C, generator=g, device="cuda") * magnitude
    y, rstd, gamma = torch.empty_like(x), torch.empty(9, device="cuda"), torch.ones(C, device="cuda")
    h = B.RmsNorm(C, eps=eps)
    h.run(x, gamma, y, 9, rstd=rstd, stream=stream())
    torch.cuda.synchronize()
    s = x.double()
    held = torch.tensor(eps, dtype=torch.float32).double().item()      # what fp32 makes of it
    rs = ((s * s).mean(1, keepdim=True) + held) ** -0.5
    least = 2.0 ** -149
    check(rstd[:, None], rs, (adds(C) + 8) / 2 * R.EPS24 * rs * 1.01 + least, "rstd")
    check(y, s * rs, ((adds(C) + 8) / 2 + 3) * 1.01 * R.EPS24 * (s * rs).abs() + least + s.abs() * least, "y")
