"""A compressed bottleneck: pattern-pruned 3x3 layer -> group norm + ReLU -> 1x1 layer with 4-bit weights, and a few steps that fine-tune
the norm's scale and shift after pruning.

    python examples/bottleneck_4bit.py

Needs a CUDA device; prints the relative error of the compressed block against the same block in fp32, and the loss before and after the
fine-tuning steps.
"""
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2001_00138_b200 import binding as pat, synth  # noqa: E402

EPS = 1e-5


def main(N=4, C=64, H=28, W=28, groups=32, out_channels=256, steps=20, lr=0.05, seed=0):
    stream = torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device="cuda").manual_seed(seed)
    P, rows = H * W, N * H * W

    # the 3x3 layer, pattern-pruned (fp16, NCHW), as everywhere in this library
    L = synth.make_layer("bottleneck", F=C, C=C, N=N, H=H, W=W, seed=seed + 1, prune=0.5, dtype="f16", draw_input=False,
                         w_std=float(np.sqrt(2.0 / (4 * C * 0.5))))
    conv = pat.encode(L.weights, L.mask, L.patterns, N=N, H=H, W=W, dtype=pat.F16, relu=False, bias=L.bias)
    x = torch.randn(N, C, H, W, generator=g, device="cuda").half()
    y = torch.empty_like(x)
    conv.conv(x, y, stream)
    pixels = y.permute(0, 2, 3, 1).reshape(N, P, C).contiguous()          # channels last: a pixel is a row

    # group norm + ReLU straight into 4-bit rows, then the 1x1 layer on them
    gamma, beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")
    norm = pat.GroupNorm(N, P, C, groups, dtype=pat.F16, act=pat.ACT_RELU, eps=EPS)
    w = (torch.randn(out_channels, C, generator=g, device="cuda") / C ** 0.5).half()
    linear = pat.Linear(w, out_channels, C, max_rows=rows, dtype=pat.F16, stream=stream)
    mx = torch.empty(pat.mx4_bytes(rows, C), dtype=torch.uint8, device="cuda")
    out = torch.empty(rows, out_channels, dtype=torch.float16, device="cuda")
    stats = torch.empty(N, groups, 2, device="cuda")
    norm.run_mx4(pixels, gamma, beta, mx, stats=stats, stream=stream)
    linear.run_mx4(mx, out, rows, stream=stream)
    conv.check()
    linear.check()

    full = torch.nn.functional.group_norm(y.float(), groups, eps=EPS).relu().permute(0, 2, 3, 1).reshape(rows, C) @ w.float().t()
    error = ((out.float() - full).norm() / full.norm()).item()

    # the values that those 4-bit rows stand for, read back
    values = torch.empty(rows, C, dtype=torch.float16, device="cuda")
    pat.mx4_dequantize(mx, values, rows, C, dtype=pat.F16, stream=stream)

    # fine-tuning after pruning: the norm's parameters towards a teacher's activations, through the norm and its gradient
    teacher_gamma = 1 + 0.3 * torch.randn(C, generator=g, device="cuda")
    teacher_beta = 0.3 * torch.randn(C, generator=g, device="cuda")
    tune = pat.GroupNorm(N, P, C, groups, dtype=pat.F16, act=pat.ACT_SILU, eps=EPS)
    target, a, d = (torch.empty(N, P, C, dtype=torch.float16, device="cuda") for _ in range(3))
    dgamma, dbeta = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    tune.run(pixels, teacher_gamma, teacher_beta, target, stream=stream)
    losses = []
    for _ in range(steps):
        tune.run(pixels, gamma, beta, a, stats=stats, stream=stream)
        off = a.float() - target.float()
        losses.append((off ** 2).mean().item())
        tune.grad(pixels, gamma, beta, stats, off.half(), d, dgamma, dbeta, stream=stream)
        gamma -= lr * 20 * dgamma / rows
        beta -= lr * 20 * dbeta / rows
    return dict(error=error, values=values, losses=losses)


if __name__ == "__main__":
    r = main()
    print(f"compressed block against fp32: relative error {r['error']:.3f}; loss {r['losses'][0]:.4f} -> {r['losses'][-1]:.4f}")
