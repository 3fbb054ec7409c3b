"""Bounded waits of the RMS norm's clusters (rows that several CTAs share): one that runs out gives NaN for its row and the rows behind it, never a wrong
number; patdnn_rms_check reports it, and the handle works again afterwards.

Nothing here faults, traps or hangs the GPU: the bound is shortened to a few milliseconds and clusters wait for a value that nobody sends (patdnn_rms_debug_wait), so that the
wait for it runs out.
"""
import pytest

from ff_ref import mx8_buffer, refused, stream, types

pytestmark = pytest.mark.gpu
E_SHAPE, E_DEVICE_TIMEOUT = 2, 8


@pytest.mark.parametrize("what", ["norm", "8 bits", "gradient"])
@pytest.mark.parametrize("M, C, dtype, skip", [(300, 16384, "bf16", 1), (300, 16384, "bf16", 3), (260, 5000, "f32", 2), (1000, 20000, "f16", 5), (100, 65536, "bf16", 4), (100, 65536, "f32", 3)])
def test_a_wait_that_runs_out_is_reported_and_the_handle_keeps_working(M, C, dtype, skip, what):
    import torch
    from paper_2001_00138_b200 import binding as B
    if what != "gradient" and C <= 8192:
        return                                             # (a CTA alone has such rows)
    tt, dt = types(dtype)
    g = torch.Generator(device="cuda").manual_seed(M + C)
    x, dy = (torch.randn(M, C, generator=g, device="cuda").to(tt) for _ in range(2))
    gamma, rstd = 1 + torch.rand(C, generator=g, device="cuda"), torch.ones(M, device="cuda")
    h, y, out, dgamma, mx = B.RmsNorm(C, dtype=dt), torch.empty_like(x), torch.empty(M, C, device="cuda"), torch.empty(C, device="cuda"), mx8_buffer(M, C)

    def step():
        if what == "norm":
            h.run(x, gamma, y, M, stream=stream())
        elif what == "gradient":
            h.grad(x, gamma, rstd, dy, y, dgamma, M, stream=stream())
        else:
            h.run_mx8(x, gamma, mx, M, stream=stream())
            B.mx8_dequantize(mx, out, M, C, stream=stream())
        torch.cuda.synchronize()
        return (out if what == "8 bits" else y).clone()

    want = step()
    h.check()
    assert torch.isfinite(want).all()
    h.debug_wait(1024, skip)
    got = step()
    refused(E_DEVICE_TIMEOUT, h.check)
    h.check()                                              # the report cleared the status word
    bad = torch.isnan(got)
    assert bad.any() and torch.equal(got[~bad], want[~bad])
    h.debug_wait(0, 0)
    assert torch.equal(step(), want)
    h.check()
    refused(E_SHAPE, h.debug_wait, 0, -1)
    h.free()


def test_a_row_of_one_cta_has_no_wait():
    import torch
    from paper_2001_00138_b200 import binding as B
    x = torch.randn(40, 4096, device="cuda")
    h, y, want, gamma = B.RmsNorm(4096), torch.empty_like(x), torch.empty_like(x), torch.ones(4096, device="cuda")
    h.run(x, gamma, want, 40, stream=stream())
    h.debug_wait(1, 1)
    h.run(x, gamma, y, 40, stream=stream())
    h.check()
    assert torch.equal(y, want)
