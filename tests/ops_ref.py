"""Plain 64-bit statements of the group norm, its gradient and the 4-bit blocks, used by the tests."""
import numpy as np

EPS24 = 2.0 ** -24                 # unit roundoff of fp32
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}    # half: half the spacing of its subnormals

_POSITIVE = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def act(z, name):
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return np.ones_like(z)


def norm(x, gamma, beta, groups, eps, name):
    """x [N][P][C] -> dict of y, z, xh, and per-channel mean and rstd [N][1][C]."""
    n, p, c = x.shape
    v = x.reshape(n, p, groups, c // groups)
    mean = v.mean(axis=(1, 3))
    var = ((v - mean[:, None, :, None]) ** 2).mean(axis=(1, 3))
    rstd = 1.0 / np.sqrt(var + eps)
    mc, rc = (np.repeat(t, c // groups, axis=1)[:, None, :] for t in (mean, rstd))
    xh = (x - mc) * rc
    z = xh * gamma + beta
    return dict(y=act(z, name), z=z, xh=xh, mean=mean, rstd=rstd, mc=mc, rc=rc)


def norm_grad(x, gamma, beta, groups, eps, name, dy):
    n, p, c = x.shape
    f = norm(x, gamma, beta, groups, eps, name)
    dz = dy * slope(f["z"], name)
    u = dz * gamma

    def group_mean(t):
        m = t.reshape(n, p, groups, -1).mean(axis=(1, 3))
        return np.repeat(m, c // groups, axis=1)[:, None, :]

    dx = f["rc"] * (u - group_mean(u) - f["xh"] * group_mean(u * f["xh"]))
    size = f["rc"] * (np.abs(u) + group_mean(np.abs(u)) + np.abs(f["xh"]) * group_mean(np.abs(u * f["xh"])))
    return dict(dx=dx, dgamma=(dz * f["xh"]).sum((0, 1)), dbeta=dz.sum((0, 1)), dx_size=size, fwd=f,
                dgamma_size=(np.abs(dz) * (np.abs(f["xh"]) + np.abs(f["mc"]) * f["rc"])).sum((0, 1)), dbeta_size=np.abs(dz).sum((0, 1)))


def quantise(x):
    """[R][K] -> the values its 4-bit blocks of 32 stand for (NaN for a block that is not finite)."""
    rows, k = x.shape
    out = np.empty((rows, k))
    for lo in range(0, k, 32):
        b = np.asarray(x[:, lo:lo + 32], dtype=np.float64)
        top = np.abs(b).max(axis=1)
        ok = np.isfinite(top)
        e = np.full(rows, -127)
        pos = ok & (top > 0)
        e[pos] = np.maximum(np.frexp(top[pos])[1] - 3, -127)
        scale = np.ldexp(np.ones(rows), e)[:, None]
        r = np.abs(np.where(ok[:, None], b, 0.0)) / scale
        d = np.abs(r[:, :, None] - _POSITIVE)
        near = d.min(axis=2, keepdims=True)
        tied = d == near                                   # at most two neighbours; the even code wins
        code = np.where(tied[:, :, ::2].any(axis=2), tied[:, :, ::2].argmax(axis=2) * 2, tied.argmax(axis=2))
        v = np.copysign(_POSITIVE[code], b) * scale
        v[~ok] = np.nan
        out[:, lo:lo + 32] = v
    return out


def within(got, ref, bound, what):
    """|got - ref| <= bound element by element."""
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    bad = ~(np.abs(got - ref) <= bound)
    if bad.any():
        i = np.unravel_index(np.argmax(np.where(bad, np.abs(got - ref) / np.maximum(bound, 1e-300), 0)), ref.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {ref.size} outside; at {i} got {got[i]}, want {ref[i]}, bound "
                             f"{np.broadcast_to(bound, ref.shape)[i]}")
