"""The feed-forward operators together, as the example runs them: the served chain and the gradients of a fine-tuning step.

The gradients are held against autograd in 64 bits.  What is rounded to bf16 on the way (2^-8 each, independent and averaged in the products):
y, gu, dg and du, dy, and the results; a tensor's relative error in norm is then at most a few of them, 8 * 2^-8, for every one of its roundings
being at most 2^-8 of the magnitude that it rounds.  The chain's 8-bit parts round by at most 2^-4 of the magnitude, three times over two
products each: 0.2 in norm would need every rounding at its worst and in the same direction.
"""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("sizes", [dict(), dict(rows=1, width=320, hidden=700, classes=33), dict(rows=70, width=130, hidden=97, classes=10)])
def test_example_runs_and_its_gradients(sizes):
    import torch
    import feed_forward_8bit as example
    r = example.main(steps=2, **sizes)
    assert torch.isfinite(r["logits"].float()).all() and r["error"] < 0.2
    t = {k: v.double() for k, v in r["gradients"].items()}
    leaf = {k: t[k].requires_grad_() for k in ("x", "gamma", "wg", "wu")}
    s = leaf["x"] + t["residual"]
    z = s * ((s * s).mean(1, keepdim=True) + example.EPS) ** -0.5 * leaf["gamma"]
    g, u = z @ leaf["wg"].t(), z @ leaf["wu"].t()
    (g * torch.sigmoid(g) * u * t["dh"]).sum().backward()
    for name, got in (("x", "dx"), ("gamma", "dgamma"), ("wg", "dwg"), ("wu", "dwu")):
        want = leaf[name].grad
        assert (t[got] - want).norm() <= 8 * 2.0 ** -8 * want.norm(), name


def test_the_chain_in_one_captured_graph():
    """Norm, block, projection and next norm captured together, replayed on other inputs: the same bits as the calls one by one."""
    import torch
    from paper_2001_00138_b200 import binding as pat
    rows, width, hidden = 33, 256, 640
    g = torch.Generator(device="cuda").manual_seed(4)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).half()

    wg, wu, down = normal(hidden, width, scale=width ** -0.5), normal(hidden, width, scale=width ** -0.5), normal(width, hidden, scale=hidden ** -0.5)
    gamma = torch.ones(width, device="cuda")
    norm = pat.RmsNorm(width, dtype=pat.F16)
    block = pat.Gated(hidden, width, max_rows=rows, dtype=pat.F16)
    back = pat.Linear8(down, width, hidden, max_rows=rows, dtype=pat.F16, stream=torch.cuda.current_stream().cuda_stream)
    x, carried = normal(rows, width), normal(rows, width)
    y, h, o, z = torch.empty_like(x), torch.empty(rows, hidden, dtype=torch.float16, device="cuda"), torch.empty_like(x), torch.empty_like(x)

    def chain(stream):
        norm.run(x, gamma, y, rows, residual=carried, sum=carried, stream=stream)
        block.run(y, wg, wu, h, rows, stream=stream)
        back.run(h, o, rows, stream=stream)
        norm.run(o, gamma, z, rows, residual=carried, sum=carried, stream=stream)

    inputs = [(normal(rows, width), normal(rows, width)) for _ in range(3)]
    wants = []
    for a, b in inputs:
        x.copy_(a)
        carried.copy_(b)
        chain(torch.cuda.current_stream().cuda_stream)
        wants.append((z.clone(), carried.clone()))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(torch.cuda.current_stream().cuda_stream)
    for (a, b), want in zip(inputs, wants):
        x.copy_(a)
        carried.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, want[0]) and torch.equal(carried, want[1])


def test_calls_on_two_streams_at_once():
    """A handle each: gradients of the block and of the norm on one stream, the block and 8-bit products on another, in turn and together."""
    import torch
    from paper_2001_00138_b200 import binding as pat
    g = torch.Generator(device="cuda").manual_seed(5)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).bfloat16()

    sides = []
    for rows, width, hidden in ((700, 512, 1100), (40, 1000, 2048)):
        x, dh, carried = normal(rows, width), normal(rows, hidden), normal(rows, width)
        wg, wu, down = normal(hidden, width, scale=width ** -0.5), normal(hidden, width, scale=width ** -0.5), normal(width, hidden, scale=hidden ** -0.5)
        gamma, rstd = torch.rand(width, generator=g, device="cuda"), torch.ones(rows, device="cuda")
        out = dict(gu=normal(rows, 2, hidden), h=dh.clone(), dx=x.clone(), dwg=wg.clone(), dwu=wu.clone(), o=x.clone(), dn=x.clone(), dgamma=gamma.clone())
        norm, block = pat.RmsNorm(width, dtype=pat.BF16), pat.Gated(hidden, width, max_rows=rows, dtype=pat.BF16, grad=True)
        back = pat.Linear8(down, width, hidden, max_rows=rows, dtype=pat.BF16, stream=torch.cuda.current_stream().cuda_stream)

        def side(st, rows=rows, x=x, dh=dh, carried=carried, wg=wg, wu=wu, gamma=gamma, rstd=rstd, o=out, norm=norm, block=block, back=back):
            block.run(x, wg, wu, o["h"], rows, gu=o["gu"], stream=st)
            back.run(o["h"], o["o"], rows, stream=st)
            block.grad(x, wg, wu, o["gu"], dh, o["dx"], o["dwg"], o["dwu"], rows, stream=st)
            norm.grad(carried, gamma, rstd, o["dx"], o["dn"], o["dgamma"], rows, dsum=o["o"], stream=st)

        sides.append((side, out, (block, back)))
    wants = []
    for side, out, _ in sides:
        side(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        wants.append({k: v.clone() for k, v in out.items()})
        for v in out.values():
            v.zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, (side, _, _) in zip(streams, sides):
            side(st.cuda_stream)
    torch.cuda.synchronize()
    for (_, out, handles), want in zip(sides, wants):
        for h in handles:
            h.check()
        for k, v in want.items():
            assert torch.isfinite(v).all() and torch.equal(out[k], v), k
