"""Measured cases of the feed-forward operators: RMS norm with the residual's addition and its gradient, 8-bit matrices with a scale per
128 columns, the linear layer with 8-bit weights (alone and behind the norm), and the gated feed-forward block with its gradient.

``run`` computes the plain form in fp32 from elementary torch operations, or (``own``) calls the library; ``exact`` states the
definitions in 64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
BLOCK = 128         # columns of a row that share one power-of-two scale


# ---------------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # serving: the residual stream of a single token, latency of a small launch
        dict(name="norm_row", kind="norm", M=1, K=4096, dtype="f16", slack=0),
        # a prompt or a training batch of 16384 tokens: memory bandwidth
        dict(name="norm_large", kind="norm", M=16384, K=4096, dtype="bf16", slack=0),
        # training in fp32, rows inside a wider tensor
        dict(name="norm_grad_f32", kind="norm_grad", M=4095, K=2560, dtype="f32", slack=4),
        # rows that are neither a multiple of the block nor of the vector width
        dict(name="quant_ragged", kind="quant", M=197, K=1001, dtype="f32", slack=3),
        # a large activation matrix
        dict(name="quant_large", kind="quant", M=16384, K=4096, dtype="bf16", slack=0),
        # serving a single token: the weights are read once
        dict(name="linear_row", kind="linear", M=1, K=4096, F=4096, dtype="f16", act="none", slack=0),
        # a compute-bound product
        dict(name="linear_large", kind="linear", M=8192, K=4096, F=4096, dtype="bf16", act="none", slack=0),
        # serving a few requests' prompts: the norm writes the 8-bit rows that the product reads
        dict(name="norm_linear_ordinary", kind="norm_linear", M=333, K=2048, F=1000, dtype="f16", act="relu", slack=0),
        # serving a single token through the gated block: two weight matrices are read once
        dict(name="gated_row", kind="gated", M=1, K=4096, F=8192, dtype="bf16", act="silu", slack=0),
        # training, forward pass, 4096 tokens
        dict(name="gated_large", kind="gated", M=4096, K=4096, F=8192, dtype="bf16", act="silu", slack=0),
        # sizes that fill no tile
        dict(name="gated_grad_ragged", kind="gated_grad", M=777, K=1000, F=1333, dtype="f16", act="silu", slack=8),
        # training, backward pass, 4096 tokens
        dict(name="gated_grad_large", kind="gated_grad", M=4096, K=2048, F=8192, dtype="bf16", act="silu", slack=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "quant", "linear", "norm_linear", "gated", "gated_grad"])
    dtype = rng.choice(["f32", "f16", "bf16"] if not kind.startswith("gated") else ["f16", "bf16"])
    slack = rng.choice([0, 0, 0, 8, 3])
    even = rng.choice([1, 1, 8, 64])                       # sizes as they come, and multiples of a vector or of a tile

    def size(lo, hi):
        return max(1, _log(rng, lo, hi) // even) * even

    k = size(20, 16384) if kind in ("norm", "norm_grad", "quant") else size(48, 8192)
    if kind in ("norm", "norm_grad", "quant"):
        return dict(kind=kind, M=_log(rng, 1, min(65536, 30_000_000 // k)), K=k, dtype=dtype, slack=slack)
    f = size(16, 8192)
    m = _log(rng, 1, min(8192, max(2, 4096 * 4096 * 2048 // (k * f))))
    return dict(kind=kind, M=m, K=k, F=f, dtype=dtype, act=rng.choice(["none", "relu", "silu"]), slack=slack)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    kind, m, k, f = case["kind"], case["M"], case["K"], case.get("F", 0)
    held = 1 + 1 / BLOCK                                   # bytes of an element held in 8 bits
    if kind == "norm":
        return {"bytes": m * (4 * k * e + 4) + 4 * k, "flops": 5 * m * k}
    if kind == "norm_grad":
        return {"bytes": m * (4 * k * e + 4) + 8 * k, "flops": 10 * m * k}
    if kind == "quant":
        return {"bytes": int(m * k * (2 * e + held)), "flops": 2 * m * k}
    if kind == "linear":
        return {"bytes": int(e * m * (k + f) + f * k * held + 4 * f), "flops": 2 * m * k * f}
    if kind == "norm_linear":
        return {"bytes": int(e * m * (3 * k + f) + f * k * held + 4 * f + 4 * k), "flops": 2 * m * k * f + 6 * m * k}
    if kind == "gated":
        return {"bytes": e * (m * (k + f) + 2 * f * k), "flops": 4 * m * k * f}
    return {"bytes": e * (m * (2 * k + 3 * f) + 4 * f * k), "flops": 8 * m * k * f}


# --------------------------------------------------------------------------------------------------------------- inputs
def _inputs(case, seed):
    """What the user's program has: tensors of the case's type, rows `slack` elements further apart than they are long."""
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)
    t, kind, m, k = TYPES[case["dtype"]], case["kind"], case["M"], case["K"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def spaced(v):
        wide = torch.zeros(*v.shape[:-1], v.shape[-1] + case["slack"], device="cuda", dtype=t)
        wide[..., : v.shape[-1]] = v
        return wide[..., : v.shape[-1]]

    d = {}
    if kind in ("norm", "norm_linear", "norm_grad"):
        # a residual stream: some columns much larger than the rest; what a layer adds to it is smaller
        stream = normal(m, k) * torch.exp(0.7 * normal(k)) * (0.5 + normal(m, 1).abs())
        d["gamma"] = 1 + 0.2 * normal(k)
        if kind == "norm_grad":
            d["s"], d["dy"], d["ds"] = spaced(stream), spaced(normal(m, k)), spaced(normal(m, k))
            d["rstd"] = _rstd(d["s"].float())              # kept from the forward pass
        else:
            d["r"], d["x"] = spaced(stream), spaced(0.5 * normal(m, k))
    if kind == "quant":
        # activations: mostly small, a few columns much larger
        d["x"] = spaced(normal(m, k) * torch.exp(normal(k)))
    if kind in ("linear", "gated", "gated_grad"):
        d["x"] = spaced(normal(m, k))
    if kind in ("linear", "norm_linear"):
        d["w"] = (normal(case["F"], k) / math.sqrt(k)).to(t)
        d["bias"] = 0.1 * normal(case["F"])
    if kind in ("gated", "gated_grad"):
        f = case["F"]
        d["wg"], d["wu"] = ((normal(f, k) / math.sqrt(k)).to(t) for _ in range(2))
        if kind == "gated_grad":
            d["dh"] = spaced(normal(m, f))
            # kept from the forward pass: both projections, in the case's type
            d["gu"] = torch.cat([(d["x"].float() @ d[w].float().t()).to(t) for w in ("wg", "wu")], dim=1)
    return d


def _rstd(s):
    return torch.rsqrt((s * s).mean(dim=-1) + EPS)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind, t, m, k = case["kind"], TYPES[case["dtype"]], case["M"], case["K"]
    if own:
        from paper_2001_00138_b200 import binding as pat
        s["pat"] = pat
        dt = {"f32": pat.F32, "f16": pat.F16, "bf16": pat.BF16}[case["dtype"]]
        act = {"none": pat.ACT_NONE, "relu": pat.ACT_RELU, "silu": pat.ACT_SILU}[case.get("act", "none")]
        s["dt"], s["stream"] = dt, torch.cuda.current_stream().cuda_stream

        def spaced(*shape):
            return torch.empty(*shape[:-1], shape[-1] + case["slack"], device="cuda", dtype=t)[..., : shape[-1]]

        if kind in ("norm", "norm_linear"):
            s["norm"] = pat.RmsNorm(k, dtype=dt, eps=EPS, x_row=s["x"].stride(0), r_row=s["r"].stride(0))
            s["sum"] = spaced(m, k)
        if kind == "norm":
            s["y"], s["rstd"] = torch.empty(m, k, device="cuda", dtype=t), torch.empty(m, device="cuda")
        if kind == "norm_grad":
            s["norm"] = pat.RmsNorm(k, dtype=dt, eps=EPS, x_row=k + case["slack"], r_row=s["s"].stride(0), y_row=s["dy"].stride(0))
            s["dx"], s["dgamma"] = spaced(m, k), torch.empty(k, device="cuda")
        if kind in ("quant", "norm_linear"):
            s["mx"] = torch.empty(pat.mx8_bytes(m, k), device="cuda", dtype=torch.uint8)
        if kind == "quant":
            s["values"] = torch.empty(m, k, device="cuda", dtype=t)
        if kind in ("linear", "norm_linear"):
            s["linear"] = pat.Linear8(s["w"], case["F"], k, max_rows=m if kind == "linear" else 0, dtype=dt, bias=s["bias"], act=act, stream=s["stream"])
            s["y"] = torch.empty(m, case["F"], device="cuda", dtype=t)
        if kind in ("gated", "gated_grad"):
            s["gated"] = pat.Gated(case["F"], k, max_rows=m, dtype=dt, act=act, x_row=s["x"].stride(0),
                                   h_row=s["dh"].stride(0) if kind == "gated_grad" else 0, grad=kind == "gated_grad")
        if kind == "gated":
            s["h"] = torch.empty(m, case["F"], device="cuda", dtype=t)
        if kind == "gated_grad":
            s["dx"], s["dwg"], s["dwu"] = spaced(m, k), torch.empty_like(s["wg"]), torch.empty_like(s["wu"])
    elif kind in ("linear", "norm_linear"):
        s["wq"] = _fake_quantize(s["w"].float())           # the layer's weights, quantised once
    return s


# ----------------------------------------------------------------------------------------------------------- plain form
def _act(z, act):
    return z.clamp_min(0) if act == "relu" else z / (1 + torch.exp(-z)) if act == "silu" else z


def _fake_quantize(x):
    """fp32 [M, K] -> the fp32 values that its 8-bit blocks stand for."""
    m, k = x.shape
    pad = -k % BLOCK
    if pad:
        x = torch.cat([x, x.new_zeros(m, pad)], dim=1)
    b = x.reshape(m, -1, BLOCK)
    f, e = torch.frexp(b.abs().amax(dim=-1, keepdim=True))             # amax = f * 2^e, 1/2 <= f < 1; 448 = 0.875 * 2^9
    exponent = (e - 9 + (f > 0.875)).clamp_min(-127)
    exponent = torch.where(f > 0, exponent, torch.full_like(exponent, -127))
    v = torch.ldexp(b, -exponent)                                      # within [-448, 448]: exact
    step = torch.ldexp(torch.ones_like(v), (torch.frexp(v)[1] - 4).clamp_min(-9))      # three bits behind the leading one
    return torch.ldexp(torch.round(v / step) * step, exponent).reshape(m, k + pad)[:, :k]


def _plain_norm(s):
    total = s["x"].float() + s["r"].float()
    rstd = _rstd(total)
    return total, rstd, total * rstd[:, None] * s["gamma"]


def _plain_gated_grad(s):
    act, f = s["case"]["act"], s["case"]["F"]
    g, u, dh = s["gu"][:, :f].float(), s["gu"][:, f:].float(), s["dh"].float()
    if act == "silu":
        sig = 1 / (1 + torch.exp(-g))
        a, slope = g * sig, sig * (1 + g * (1 - sig))
    elif act == "relu":
        a, slope = g.clamp_min(0), (g > 0).float()
    else:
        a, slope = g, torch.ones_like(g)
    dg, du, x = dh * u * slope, dh * a, s["x"].float()
    return dg @ s["wg"].float() + du @ s["wu"].float(), dg.t() @ x, du.t() @ x


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        return _run_own(s, kind, case)
    t = TYPES[case["dtype"]]
    if kind == "norm":
        total, rstd, y = _plain_norm(s)
        return {"y": y.to(t), "sum": total.to(t), "rstd": rstd}
    if kind == "norm_grad":
        xh, u = s["s"].float() * s["rstd"][:, None], s["dy"].float() * s["gamma"]
        dx = s["rstd"][:, None] * (u - xh * (u * xh).mean(dim=1, keepdim=True)) + s["ds"].float()
        return {"dx": dx.to(t), "dgamma": (s["dy"].float() * xh).sum(dim=0)}
    if kind == "quant":
        return {"values": _fake_quantize(s["x"].float()).to(t)}
    if kind == "linear":
        y = _fake_quantize(s["x"].float()) @ s["wq"].t() + s["bias"]
        return {"y": _act(y, case["act"]).to(t)}
    if kind == "norm_linear":
        total, _, z = _plain_norm(s)
        y = _fake_quantize(z) @ s["wq"].t() + s["bias"]
        return {"y": _act(y, case["act"]).to(t), "sum": total.to(t)}
    if kind == "gated":
        x = s["x"].float()
        return {"h": (_act(x @ s["wg"].float().t(), case["act"]) * (x @ s["wu"].float().t())).to(t)}
    dx, dwg, dwu = _plain_gated_grad(s)
    return {"dx": dx.to(t), "dwg": dwg.to(t), "dwu": dwu.to(t)}


def _run_own(s, kind, case):
    stream, pat, m, k = s["stream"], s["pat"], case["M"], case["K"]
    if kind == "norm":
        s["norm"].run(s["x"], s["gamma"], s["y"], m, residual=s["r"], sum=s["sum"], rstd=s["rstd"], stream=stream)
        return {"y": s["y"], "sum": s["sum"], "rstd": s["rstd"]}
    if kind == "norm_grad":
        s["norm"].grad(s["s"], s["gamma"], s["rstd"], s["dy"], s["dx"], s["dgamma"], m, dsum=s["ds"], stream=stream)
        return {"dx": s["dx"], "dgamma": s["dgamma"]}
    if kind == "quant":
        pat.mx8_quantize(s["x"], s["mx"], m, k, dtype=s["dt"], ld=s["x"].stride(0), stream=stream)
        pat.mx8_dequantize(s["mx"], s["values"], m, k, dtype=s["dt"], stream=stream)
        return {"values": s["values"]}
    if kind == "linear":
        s["linear"].run(s["x"], s["y"], m, ldx=s["x"].stride(0), stream=stream)
        return {"y": s["y"]}
    if kind == "norm_linear":
        s["norm"].run_mx8(s["x"], s["gamma"], s["mx"], m, residual=s["r"], sum=s["sum"], stream=stream)
        s["linear"].run_mx8(s["mx"], s["y"], m, stream=stream)
        return {"y": s["y"], "sum": s["sum"]}
    if kind == "gated":
        s["gated"].run(s["x"], s["wg"], s["wu"], s["h"], m, stream=stream)
        return {"h": s["h"]}
    s["gated"].grad(s["x"], s["wg"], s["wu"], s["gu"], s["dh"], s["dx"], s["dwg"], s["dwu"], m, stream=stream)
    return {"dx": s["dx"], "dwg": s["dwg"], "dwu": s["dwu"]}


# --------------------------------------------------------------------------------------------------- 64-bit definitions
# the magnitudes of eight bits with four for the exponent: seven of 2^-9 apart below 2^-6, then eight to an octave up to 448
_GRID = [i * 2.0 ** -9 for i in range(8)] + [(1 + i / 8) * 2.0 ** e for e in range(-6, 9) for i in range(8)][:-1]


def _nearest64(x):
    """The value each element of a float64 matrix takes when its blocks of 128 are held in 8 bits: the scale is the smallest power of two
    at which the block's largest magnitude is at most 448; then the nearest magnitude of the grid, the one of even code at a tie."""
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
        power = ((top.view(torch.int64) >> 52) - 1023 - 8).double()         # 256 to 512 times this power of two
        scale = torch.exp2(torch.where(top > 448 * torch.exp2(power), power + 1, power).clamp_min(-127))
        scale = torch.where(top > 0, scale, torch.ones_like(top))
        r = b.abs() / scale
        below = torch.bucketize(r, middle)                 # middles that lie strictly under r
        tie = (below < len(_GRID) - 1) & (r == middle[below.clamp_max(len(_GRID) - 2)])
        code = torch.where(tie & (below % 2 == 1), below + 1, below)
        out[:, lo:hi] = (torch.copysign(grid[code], b) * scale).reshape(m, hi - lo)
    return out


def exact(case, seed):
    d = {n: v.double() for n, v in _inputs(case, seed).items()}
    kind, act = case["kind"], case.get("act")

    def activate(z):
        return z.relu() if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z

    if kind == "quant":
        return {"values": _nearest64(d["x"])}
    if kind == "linear":
        return {"y": activate(torch.addmm(d["bias"], _nearest64(d["x"]), _nearest64(d["w"]).t()))}
    if kind in ("norm", "norm_linear"):
        total = d["x"] + d["r"]
        length = torch.linalg.vector_norm(total, dim=1)
        rstd = (length.square() / case["K"] + EPS) ** -0.5
        z = torch.einsum("mk,m,k->mk", total, rstd, d["gamma"])
        if kind == "norm":
            return {"y": z, "sum": total, "rstd": rstd}
        return {"y": activate(torch.addmm(d["bias"], _nearest64(z), _nearest64(d["w"]).t())), "sum": total}
    if kind == "norm_grad":
        u = d["dy"] * d["gamma"]
        along = torch.einsum("mk,mk->m", u, d["s"]) * d["rstd"] ** 3 / case["K"]
        return {"dx": u * d["rstd"][:, None] - d["s"] * along[:, None] + d["ds"],
                "dgamma": torch.einsum("mk,mk,m->k", d["dy"], d["s"], d["rstd"])}
    if kind == "gated":
        return {"h": activate(d["x"].matmul(d["wg"].t())).mul_(d["x"].matmul(d["wu"].t()))}
    g, u = d["gu"].split(case["F"], dim=1)
    sg = torch.sigmoid(g)
    slope = sg + g * sg * (1 - sg) if act == "silu" else (g > 0).double() if act == "relu" else torch.ones_like(g)
    dgu = torch.cat([d["dh"] * u * slope, d["dh"] * activate(g)], dim=1)
    dw = dgu.t().matmul(d["x"])
    return {"dx": dgu.matmul(torch.cat([d["wg"], d["wu"]])), "dwg": dw[: case["F"]], "dwu": dw[case["F"]:]}
