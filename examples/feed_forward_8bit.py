"""A feed-forward part of a network, served and fine-tuned: RMS norm that adds the residual -> gated block -> projection back with 8-bit weights
-> next norm, whose 8-bit rows go straight into a head with 8-bit weights; and a few steps that fit the gated block and the norm's scale to a
teacher's hidden values, with the gradients of both.

    python examples/feed_forward_8bit.py

Needs a CUDA device; prints the relative error of the served chain against the same chain in fp32, and the loss before and after the steps.
"""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2001_00138_b200 import binding as pat  # noqa: E402

EPS = 1e-6


def main(rows=256, width=512, hidden=1408, classes=1000, steps=10, lr=0.02, seed=0):
    stream = torch.cuda.current_stream().cuda_stream
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).bfloat16()

    wg, wu, down, head = normal(hidden, width, scale=width ** -0.5), normal(hidden, width, scale=width ** -0.5), normal(width, hidden, scale=hidden ** -0.5), normal(classes, width, scale=width ** -0.5)
    x, residual = normal(rows, width, scale=0.5), normal(rows, width)
    gamma = 1 + 0.1 * torch.randn(width, generator=g, device="cuda")

    # serving: four calls; the residual stream is updated in its own buffer
    norm = pat.RmsNorm(width, dtype=pat.BF16, eps=EPS)
    block = pat.Gated(hidden, width, max_rows=rows, dtype=pat.BF16, act=pat.ACT_SILU, grad=True)
    back = pat.Linear8(down, width, hidden, max_rows=rows, dtype=pat.BF16, stream=stream)
    scores = pat.Linear8(head, classes, width, max_rows=0, dtype=pat.BF16, stream=stream)       # is given 8-bit rows only
    carried = residual.clone()
    y, h, o = torch.empty_like(x), torch.empty(rows, hidden, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x)
    logits = torch.empty(rows, classes, dtype=torch.bfloat16, device="cuda")
    mx = torch.empty(pat.mx8_bytes(rows, width), dtype=torch.uint8, device="cuda")
    norm.run(x, gamma, y, rows, residual=carried, sum=carried, stream=stream)
    block.run(y, wg, wu, h, rows, stream=stream)
    back.run(h, o, rows, stream=stream)
    norm.run_mx8(o, gamma, mx, rows, residual=carried, sum=carried, stream=stream)
    scores.run_mx8(mx, logits, rows, stream=stream)
    block.check()
    back.check()
    scores.check()

    def rms(v):
        return v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS) * gamma

    s = x.float() + residual.float()
    z = rms(s)
    s = s + (torch.nn.functional.silu(z @ wg.float().t()) * (z @ wu.float().t())) @ down.float().t()
    full = rms(s) @ head.float().t()
    error = ((logits.float() - full).norm() / full.norm()).item()

    # fine-tuning: the hidden values towards a teacher's
    target = h + normal(rows, hidden, scale=0.05)
    total, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    gu, dh = torch.empty(rows, 2, hidden, dtype=torch.bfloat16, device="cuda"), None
    dy, dwg, dwu, dx = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu), torch.empty_like(x)
    dgamma = torch.empty(width, device="cuda")
    losses, gradients = [], None
    for step in range(steps):
        norm.run(x, gamma, y, rows, residual=residual, sum=total, rstd=rstd, stream=stream)
        block.run(y, wg, wu, h, rows, gu=gu, stream=stream)
        off = h.float() - target.float()
        losses.append((off ** 2).mean().item())
        dh = (off * (2 / rows)).bfloat16()
        block.grad(y, wg, wu, gu, dh, dy, dwg, dwu, rows, stream=stream)
        norm.grad(total, gamma, rstd, dy, dx, dgamma, rows, stream=stream)
        if step == 0:
            gradients = dict(x=x.clone(), residual=residual.clone(), gamma=gamma.clone(), wg=wg.clone(), wu=wu.clone(), dh=dh.clone(), dwg=dwg.clone(), dwu=dwu.clone(),
                             dgamma=dgamma.clone(), dx=dx.clone())
        wg -= lr * dwg
        wu -= lr * dwu
        gamma -= lr * dgamma
    return dict(error=error, losses=losses, logits=logits, gradients=gradients)


if __name__ == "__main__":
    r = main()
    print(f"served chain against fp32: relative error {r['error']:.3f}; loss {r['losses'][0]:.5f} -> {r['losses'][-1]:.5f}")
