"""8-bit matrices read back into another type than they were quantised from: every value is the float value rounded once."""
import pytest

from ff_ref import mx8_buffer, stream, types

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [-140, -133, -130, -127, -120, -20, 0, 15, 120])
@pytest.mark.parametrize("rows, cols", [(3, 130), (200, 1000), (40, 60)])
def test_other_types(rows, cols, power):
    import torch
    from paper_2001_00138_b200 import binding as B
    g = torch.Generator().manual_seed(rows + power)
    x = torch.ldexp(torch.randn(rows, cols, generator=g) * torch.exp2(torch.randint(-9, 1, (rows, cols), generator=g).float()), torch.tensor(power)).cuda()
    mx = mx8_buffer(rows, cols)
    B.mx8_quantize(x, mx, rows, cols, stream=stream())
    outs = {}
    for dtype in ("f32", "f16", "bf16"):
        tt, dt = types(dtype)
        outs[dtype] = torch.full((rows, cols), float("nan"), dtype=tt, device="cuda")
        B.mx8_dequantize(mx, outs[dtype], rows, cols, dtype=dt, stream=stream())
    torch.cuda.synchronize()
    full = outs["f32"].cpu()
    assert torch.isfinite(full).all()
    for dtype in ("f16", "bf16"):
        assert torch.equal(outs[dtype].cpu(), full.to(types(dtype)[0])), dtype
    large = full.abs() >= 2.0 ** -130
    assert torch.equal(outs["bf16"].cpu().float()[large], full[large])
