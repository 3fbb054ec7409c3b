"""Plain 64-bit statements of the 8-bit blocks, and helpers of the feed-forward operators' tests."""
import numpy as np

from ops_ref import EPS24, TINY, UNIT, act, slope, within  # noqa: F401

BLOCK = 128
# E4M3 magnitudes by code: exponent 0 holds multiples of 2^-9, code 127 is NaN
GRID = np.array([m / 512 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])
MIDDLE = (GRID[1:] + GRID[:-1]) / 2


def quantise8(x):
    """[R][K] float64 -> the values that its 8-bit blocks of 128 stand for (NaN for a block that is not finite)."""
    rows, k = x.shape
    out = np.empty((rows, k))
    for lo in range(0, k, BLOCK):
        b = np.asarray(x[:, lo:lo + BLOCK], dtype=np.float64)
        top = np.abs(b).max(axis=1)
        ok = np.isfinite(top)
        e = np.full(rows, -127)
        pos = ok & (top > 0)
        f, p = np.frexp(top[pos] / 448.0)                  # the smallest power of two that is at least top / 448
        e[pos] = np.maximum(np.where(f == 0.5, p - 1, p), -127)
        scale = np.ldexp(np.ones(rows), e)[:, None]
        r = np.abs(np.where(ok[:, None], b, 0.0)) / scale
        code = np.searchsorted(MIDDLE, r, side="left")     # middles strictly below r
        tie = (code < 126) & (r == MIDDLE[np.minimum(code, 125)]) & (code % 2 == 1)
        v = np.copysign(GRID[np.where(tie, code + 1, code)], b) * scale
        v[~ok] = np.nan
        out[:, lo:lo + BLOCK] = v
    return out


def types(dtype):
    import torch
    from paper_2001_00138_b200 import binding as B
    return {"f32": (torch.float32, B.F32), "f16": (torch.float16, B.F16), "bf16": (torch.bfloat16, B.BF16)}[dtype]


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def mx8_buffer(rows, cols, fill=255):
    """An 8-bit matrix's buffer full of codes (NaN) and scales (NaN) that are wrong where nothing writes them."""
    import torch
    from paper_2001_00138_b200 import binding as B
    return torch.full((max(16, B.mx8_bytes(rows, cols)),), fill, dtype=torch.uint8, device="cuda")


def spaced(v, slack=0, offset=0):
    """v [R][C] with rows C + slack apart inside a tensor of NaNs, `offset` elements behind its start: (whole tensor, view)."""
    import torch
    r, c = v.shape
    flat = torch.full((offset + r * (c + slack) + 16,), float("nan"), dtype=v.dtype, device="cuda")
    view = torch.as_strided(flat, (r, c), (c + slack, 1), offset)
    view.copy_(v)
    return flat, view


def untouched(flat, *views):
    """Everything of `flat` outside the views is NaN still."""
    import torch
    inside = torch.zeros_like(flat, dtype=torch.bool)
    for v in views:
        torch.as_strided(inside, v.shape, v.stride(), v.storage_offset()).fill_(True)
    return bool(torch.isnan(flat[~inside]).all())


def refused(status, call, *args, **kw):
    import pytest
    from paper_2001_00138_b200 import binding as B
    with pytest.raises(B.PatdnnError) as e:
        call(*args, **kw)
    assert e.value.status == status, e.value


def held8(rows, cols, g):
    """Values that blocks of 128 hold exactly: whole numbers up to 15, both signs, times a power of two per block."""
    import torch
    v = torch.randint(-15, 16, (rows, cols), generator=g, device="cuda").float()
    e = torch.randint(-3, 4, (rows, -(-cols // BLOCK)), generator=g, device="cuda").repeat_interleave(BLOCK, 1)[:, :cols]
    return torch.ldexp(v, e)


def product_bound(K, size, ref, dtype):
    """The fp32 sum of an 8-bit product, 32 columns at a time: (K / 32 + 10) roundings (counted as truncations, 2^-23) of sum |x| |w| + |bias|, a
    tenth more for the activation's slope (SiLU's is at most 1.1); then the output's own rounding."""
    return 1.1 * (K / 32 + 10) * 2.0 ** -23 * size + UNIT[dtype] * abs(ref) * 1.01 + TINY[dtype]
