"""Measured cases of the operators around the pattern-pruned convolutions: group norm with an activation (channels last) and its
gradient, microscaled 4-bit quantisation, the 4-bit linear layer, and a group norm that feeds a 4-bit linear layer.

``run`` computes the plain form in fp32 from elementary torch operations, or (``own``) calls the library; ``exact`` states the
definitions in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
BLOCK = 32          # elements that share one power-of-two scale


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the 7x7 layer at the end of a ResNet-50 shaped network, one image: latency of a small launch
        dict(name="norm_tail_7x7", kind="norm", N=1, P=49, C=512, G=32, dtype="f16", act="relu", slack=0),
        # a decoder-sized image whose statistics need more than one pass over what fits on chip
        dict(name="norm_wide_512x512", kind="norm", N=2, P=512 * 512, C=128, G=32, dtype="bf16", act="silu", slack=0),
        # fine-tuning: ten channels per group, an odd image, pixels inside a wider tensor
        dict(name="grad_ragged_27x31", kind="grad", N=5, P=27 * 31, C=320, G=32, dtype="f32", act="silu", slack=12),
        # fine-tuning at batch 32 on the 56x56 stage, 256 channels
        dict(name="grad_stage_56x56", kind="grad", N=32, P=56 * 56, C=256, G=32, dtype="bf16", act="silu", slack=0),
        # rows that are neither a multiple of the block nor of the vector width
        dict(name="quant_ragged", kind="quant", M=197, K=1001, dtype="f32", slack=3),
        # a large activation matrix
        dict(name="quant_large", kind="quant", M=16384, K=4096, dtype="bf16", slack=0),
        # the second fully connected layer of a VGG-16 classifier, one image
        dict(name="linear_fc2_row", kind="linear", M=1, K=4096, F=4096, dtype="f16", act="relu", slack=0),
        # the first fully connected layer of the same classifier, batch 32: all of its weights are read
        dict(name="linear_fc1_batch32", kind="linear", M=32, K=25088, F=4096, dtype="f16", act="relu", slack=0),
        # sizes that fill no tile
        dict(name="linear_ragged", kind="linear", M=777, K=1000, F=1333, dtype="f32", act="none", slack=8),
        # a compute-bound product
        dict(name="linear_large", kind="linear", M=8192, K=4096, F=4096, dtype="bf16", act="none", slack=0),
        # the 1x1 layer behind a normalised 3x3 layer of a bottleneck, one 28x28 image
        dict(name="norm_linear_28x28", kind="norm_linear", N=1, P=28 * 28, C=128, G=32, F=512, dtype="f16", act="relu", slack=0),
        # the same at 56x56, batch 32
        dict(name="norm_linear_56x56", kind="norm_linear", N=32, P=56 * 56, C=64, G=32, F=256, dtype="bf16", act="relu", slack=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "grad", "quant", "linear", "norm_linear"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    slack = rng.choice([0, 0, 0, 8, 3])
    if kind in ("norm", "grad", "norm_linear"):
        cg = rng.choice([1, 2, 3, 4, 6, 8, 10, 12, 16, 20, 32])
        groups = rng.choice([1, 8, 16, 32, 32, 32]) if cg > 1 else rng.choice([32, 64])
        c = cg * groups
        n = _log(rng, 1, 32)
        most = {"norm": 30_000_000, "grad": 12_000_000, "norm_linear": 6_000_000}[kind]
        p = _log(rng, 4, max(5, min(512 * 512, most // (n * c))))
        act = rng.choice(["none", "relu", "silu"]) if kind != "grad" else rng.choice(["none", "silu"])
        case = dict(kind=kind, N=n, P=p, C=c, G=groups, dtype=dtype, act=act, slack=slack)
        if kind == "norm_linear":
            case["F"] = _log(rng, 16, 1024)
        return case
    if kind == "quant":
        k = _log(rng, 20, 16384)
        return dict(kind=kind, M=_log(rng, 1, min(65536, 30_000_000 // k)), K=k, dtype=dtype, slack=slack)
    k, f = _log(rng, 48, 8192), _log(rng, 16, 8192)
    m = _log(rng, 1, min(8192, max(2, 4096 * 4096 * 2048 // (k * f))))
    return dict(kind=kind, M=m, K=k, F=f, dtype=dtype, act=rng.choice(["none", "relu", "silu"]), slack=slack)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    if kind in ("norm", "grad"):
        n = case["N"] * case["P"] * case["C"]
        return {"bytes": n * e * (2 if kind == "norm" else 3) + 16 * case["C"], "flops": n * (8 if kind == "norm" else 20)}
    mx = BLOCK // 2 + 1                                   # bytes of a block: 32 codes of 4 bits and one scale
    if kind == "quant":
        return {"bytes": case["M"] * (2 * e * case["K"] + mx * -(-case["K"] // BLOCK)), "flops": 2 * case["M"] * case["K"]}
    m, k = (case["M"], case["K"]) if kind == "linear" else (case["N"] * case["P"], case["C"])
    f = case["F"]
    extra = 0 if kind == "linear" else 8 * m * k
    return {"bytes": e * m * (k + f) + f * mx * -(-k // BLOCK) + 4 * f, "flops": 2 * m * k * f + extra}


# --------------------------------------------------------------------------------------------------------------- inputs
def _inputs(case, seed):
    """What the user's program has: tensors of the case's type, rows `slack` elements further apart than they are long."""
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)
    t, kind = TYPES[case["dtype"]], case["kind"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def spaced(v):
        wide = torch.zeros(*v.shape[:-1], v.shape[-1] + case["slack"], device="cuda", dtype=t)
        wide[..., : v.shape[-1]] = v
        return wide[..., : v.shape[-1]]

    d = {}
    if kind in ("norm", "grad", "norm_linear"):
        n, p, c = case["N"], case["P"], case["C"]
        # outputs of a convolution with a bias: every channel has its own mean and spread
        d["x"] = spaced(normal(n, p, c) * (0.5 + normal(c).abs()) + normal(c))
        d["gamma"], d["beta"] = 1 + 0.1 * normal(c), 0.1 * normal(c)
        if kind == "grad":
            d["dy"] = spaced(normal(n, p, c))
    if kind == "quant":
        # activations: mostly small, a few columns much larger
        d["x"] = spaced(normal(case["M"], case["K"]) * torch.exp(normal(case["K"])))
    if kind == "linear":
        d["x"] = spaced(normal(case["M"], case["K"]).relu_() * 1.5)
    if kind in ("linear", "norm_linear"):
        k = d["x"].shape[-1]
        d["w"] = (normal(case["F"], k) / math.sqrt(k)).to(t)
        d["bias"] = 0.1 * normal(case["F"])
    return d


def _stats(x, groups):
    """Mean and 1/sqrt(var + eps) of every (image, group), fp32 [N, G, 2]."""
    n, p, c = x.shape
    v = x.float().reshape(n, p, groups, c // groups)
    mean = v.mean(dim=(1, 3), keepdim=True)
    var = ((v - mean) ** 2).mean(dim=(1, 3))
    return torch.stack([mean.reshape(n, groups), torch.rsqrt(var + EPS)], dim=-1)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind, t = case["kind"], TYPES[case["dtype"]]
    if kind == "grad":
        s["stats"] = _stats(s["x"], case["G"])            # kept from the forward pass
    if own:
        from paper_2001_00138_b200 import binding as pat
        s["pat"] = pat
        dt = {"f32": pat.F32, "f16": pat.F16, "bf16": pat.BF16}[case["dtype"]]
        act = {"none": pat.ACT_NONE, "relu": pat.ACT_RELU, "silu": pat.ACT_SILU}[case.get("act", "none")]
        s["dt"], s["stream"] = dt, torch.cuda.current_stream().cuda_stream
        x = s["x"]
        if kind in ("norm", "grad", "norm_linear"):
            n, p, c = x.shape
            s["norm"] = pat.GroupNorm(n, p, c, case["G"], dtype=dt, act=act, eps=EPS, x_pixel=x.stride(1), x_image=x.stride(0))
        if kind == "norm":
            s["y"] = torch.empty(x.shape, device="cuda", dtype=t)
            s["stats"] = torch.empty(n, case["G"], 2, device="cuda")
        if kind == "grad":
            s["norm"] = pat.GroupNorm(n, p, c, case["G"], dtype=dt, act=act, eps=EPS, x_pixel=x.stride(1), x_image=x.stride(0),
                                      y_pixel=s["dy"].stride(1), y_image=s["dy"].stride(0))
            wide = torch.empty(n, p, c + case["slack"], device="cuda", dtype=t)
            s["dx"] = wide[..., :c]
            s["dgamma"], s["dbeta"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        if kind == "quant":
            s["mx"] = torch.empty(pat.mx4_bytes(case["M"], case["K"]), device="cuda", dtype=torch.uint8)
            s["values"] = torch.empty(x.shape, device="cuda", dtype=t)
        if kind in ("linear", "norm_linear"):
            rows = x.shape[0] if kind == "linear" else n * p
            k = x.shape[-1]
            s["linear"] = pat.Linear(s["w"], case["F"], k, max_rows=rows, dtype=dt, bias=s["bias"],
                                     act=act if kind == "linear" else pat.ACT_NONE, stream=s["stream"])
            s["y"] = torch.empty(rows, case["F"], device="cuda", dtype=t)
            if kind == "norm_linear":
                s["mx"] = torch.empty(pat.mx4_bytes(rows, k), device="cuda", dtype=torch.uint8)
    elif kind in ("linear", "norm_linear"):
        s["wq"] = _fake_quantize(s["w"].float())          # the layer's weights, quantised once
    return s


# ----------------------------------------------------------------------------------------------------------- plain form
def _act(z, act):
    return z.clamp_min(0) if act == "relu" else z / (1 + torch.exp(-z)) if act == "silu" else z


def _fake_quantize(x):
    """fp32 [M, K] -> the fp32 values that its 4-bit blocks stand for."""
    m, k = x.shape
    pad = -k % BLOCK
    if pad:
        x = torch.cat([x, x.new_zeros(m, pad)], dim=1)
    b = x.reshape(m, -1, BLOCK)
    amax = b.abs().amax(dim=-1, keepdim=True)
    exponent = (torch.frexp(amax)[1] - 3).clamp_min(-127)              # amax = f * 2^e, 1/2 <= f < 1
    exponent = torch.where(amax > 0, exponent, torch.full_like(exponent, -127))
    v = torch.ldexp(b, -exponent)                                      # within (-8, 8): exact
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp_max(6) * torch.sign(v)
    return torch.ldexp(q, exponent).reshape(m, k + pad)[:, :k]


def _plain_norm(s):
    case = s["case"]
    n, p, c = s["x"].shape
    stats = _stats(s["x"], case["G"])
    v = s["x"].float().reshape(n, p, case["G"], -1)
    xh = ((v - stats[:, None, :, 0:1]) * stats[:, None, :, 1:2]).reshape(n, p, c)
    return _act(xh * s["gamma"] + s["beta"], case["act"]), stats


def _plain_grad(s):
    case, stats = s["case"], s["stats"]
    n, p, c = s["x"].shape
    groups = case["G"]
    mean, rstd = stats[:, None, :, 0:1], stats[:, None, :, 1:2]
    xh = (s["x"].float().reshape(n, p, groups, -1) - mean) * rstd
    dz = s["dy"].float()
    if case["act"] == "silu":
        z = xh.reshape(n, p, c) * s["gamma"] + s["beta"]
        sig = 1 / (1 + torch.exp(-z))
        dz = dz * sig * (1 + z * (1 - sig))
    elif case["act"] == "relu":
        dz = dz * (xh.reshape(n, p, c) * s["gamma"] + s["beta"] > 0)
    dgamma, dbeta = (dz * xh.reshape(n, p, c)).sum(dim=(0, 1)), dz.sum(dim=(0, 1))
    u = (dz * s["gamma"]).reshape(n, p, groups, -1)
    dx = rstd * (u - u.mean(dim=(1, 3), keepdim=True) - xh * (u * xh).mean(dim=(1, 3), keepdim=True))
    return dx.reshape(n, p, c), dgamma, dbeta


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _run_own(s, kind, case)
    t = TYPES[case["dtype"]]
    if kind == "norm":
        y, stats = _plain_norm(s)
        return {"y": y.to(t), "stats": stats}
    if kind == "grad":
        dx, dgamma, dbeta = _plain_grad(s)
        return {"dx": dx.to(t), "dgamma": dgamma, "dbeta": dbeta}
    if kind == "quant":
        return {"values": _fake_quantize(s["x"].float()).to(t)}
    if kind == "linear":
        y = _fake_quantize(s["x"].float()) @ s["wq"].t() + s["bias"]
        return {"y": _act(y, case["act"]).to(t)}
    z, _ = _plain_norm(s)
    return {"y": (_fake_quantize(z.reshape(-1, z.shape[-1])) @ s["wq"].t() + s["bias"]).to(t)}


def _run_own(s, kind, case):
    x, stream, pat = s["x"], s["stream"], s["pat"]
    if kind == "norm":
        s["norm"].run(x, s["gamma"], s["beta"], s["y"], stats=s["stats"], stream=stream)
        return {"y": s["y"], "stats": s["stats"]}
    if kind == "grad":
        s["norm"].grad(x, s["gamma"], s["beta"], s["stats"], s["dy"], s["dx"], s["dgamma"], s["dbeta"], stream=stream)
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if kind == "quant":
        m, k = x.shape
        pat.mx4_quantize(x, s["mx"], m, k, dtype=s["dt"], ld=x.stride(0), stream=stream)
        pat.mx4_dequantize(s["mx"], s["values"], m, k, dtype=s["dt"], stream=stream)
        return {"values": s["values"]}
    if kind == "linear":
        s["linear"].run(x, s["y"], x.shape[0], ldx=x.stride(0), stream=stream)
        return {"y": s["y"]}
    s["norm"].run_mx4(x, s["gamma"], s["beta"], s["mx"], stream=stream)
    s["linear"].run_mx4(s["mx"], s["y"], x.shape[0] * x.shape[1], stream=stream)
    return {"y": s["y"]}


# --------------------------------------------------------------------------------------------------- 64-bit definitions
_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _nearest64(x):
    """The value each element of a float64 matrix takes when its blocks of 32 are held in 4 bits: the block's largest magnitude
    gives the scale 2^(floor(log2) - 2); then the nearest of the eight magnitudes, the one of even code at a tie."""
    m, k = x.shape
    out = torch.empty_like(x)
    grid = torch.tensor(_GRID, dtype=torch.float64, device=x.device)
    middle = (grid[1:] + grid[:-1]) / 2
    full = k // BLOCK * BLOCK
    for lo, hi, width in ((0, full, BLOCK), (full, k, k - full)):
        if hi == lo:
            continue
        b = x[:, lo:hi].reshape(m, -1, width)
        top = b.abs().max(dim=-1, keepdim=True).values
        bits = (top.view(torch.int64) >> 52) - 2            # exponent field of a float64, two lower
        scale = torch.where(top > 0, (bits << 52).view(torch.float64), torch.ones_like(top))
        r = b.abs() / scale
        below = torch.bucketize(r, middle)                 # middles that lie strictly under r
        tie = (below < 7) & (r == middle[below.clamp_max(6)])
        code = torch.where(tie & (below % 2 == 1), below + 1, below)
        out[:, lo:hi] = (torch.copysign(grid[code], b) * scale).reshape(m, hi - lo)
    return out


def exact(case, seed):
    d = _inputs(case, seed)
    kind = case["kind"]
    x = d["x"].double()
    sigmoid = torch.sigmoid
    if kind == "quant":
        return {"values": _nearest64(x)}
    if kind == "linear":
        y = torch.addmm(d["bias"].double(), _nearest64(x), _nearest64(d["w"].double()).t())
        return {"y": y.relu() if case["act"] == "relu" else y * sigmoid(y) if case["act"] == "silu" else y}
    n, p, c = x.shape
    groups = case["G"]
    by = x.reshape(n, p, groups, c // groups).transpose(1, 2).reshape(n, groups, -1)
    var, mean = torch.var_mean(by, dim=2, correction=0)
    rstd = (var + EPS) ** -0.5
    per = c // groups
    mean_c, rstd_c = mean.repeat_interleave(per, 1)[:, None], rstd.repeat_interleave(per, 1)[:, None]
    del by
    xh = (x - mean_c) * rstd_c
    gamma, beta = d["gamma"].double(), d["beta"].double()
    z = torch.addcmul(beta, xh, gamma)
    if kind == "grad":
        dz = d["dy"].double()
        if case["act"] == "silu":
            sg = sigmoid(z)
            dz = dz * (sg + z * sg * (1 - sg))
        elif case["act"] == "relu":
            dz = torch.where(z > 0, dz, torch.zeros_like(dz))
        a, b = dz.sum(1), (dz * xh).sum(1)                 # [N, C]
        count = p * per
        s1 = ((a * gamma).reshape(n, groups, per).sum(2) / count).repeat_interleave(per, 1)[:, None]
        s2 = ((b * gamma).reshape(n, groups, per).sum(2) / count).repeat_interleave(per, 1)[:, None]
        return {"dx": rstd_c * (gamma * dz - s1 - xh * s2), "dgamma": b.sum(0), "dbeta": a.sum(0)}
    z = z.relu_() if case["act"] == "relu" else z * sigmoid(z) if case["act"] == "silu" else z
    if kind == "norm":
        return {"y": z, "stats": torch.stack([mean, rstd], dim=-1)}
    return {"y": torch.addmm(d["bias"].double(), _nearest64(z.reshape(-1, c)), _nearest64(d["w"].double()).t())}
