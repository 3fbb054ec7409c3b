"""Bounded waits of the linear layer's kernels: one that runs out ends the kernel through its normal exit, patdnn_linear_check reports it, and the
handle works again afterwards.

Nothing here faults, traps or hangs the GPU: the bound is shortened to a few milliseconds and the copies of one column tile are left out
(patdnn_linear_debug_wait), so that the consumers' wait for them runs out.
"""
import pytest

pytestmark = pytest.mark.gpu
E_DEVICE_TIMEOUT = 8


def make(F, K, rows, dtype="bf16", seed=0, **kw):
    """Layer, rows and buffers with whole numbers in them, whose products are exact."""
    import torch
    from paper_2001_00138_b200 import binding as B
    tt, dt = {"f32": (torch.float32, B.F32), "f16": (torch.float16, B.F16), "bf16": (torch.bfloat16, B.BF16)}[dtype]
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, w = (torch.randint(-4, 5, (n, K), generator=g, device="cuda").to(tt) for n in (rows, F))
    st = torch.cuda.current_stream().cuda_stream
    lin = B.Linear(w, F, K, max_rows=rows, dtype=dt, stream=st, **kw)
    return lin, x, w, torch.full((rows, F), float("nan"), dtype=tt, device="cuda"), st


FORMS = {  # rows, K, F, column tile that is left out, what patdnn_linear_plan has to say
    "quantises its rows": (3, 300, 100, 1, dict(quantises=1, splits=2)),
    "quantises its rows, one tile": (8, 60, 30000, 1, dict(quantises=1, splits=1)),
    "a cluster of eight": (40, 8192, 256, 3, dict(persistent=0, quantises=0, splits=8)),
    "no cluster, ring wraps": (300, 3500, 700, 9, dict(persistent=0, splits=1, column_tiles=14)),
    "many rows, 128 outputs": (20000, 300, 100, 2, dict(persistent=1, tile_outputs=128)),
    "many rows, 256 outputs, third tile": (20000, 520, 513, 8, dict(persistent=1, tile_outputs=256, column_tiles=3)),
}


@pytest.mark.parametrize("form", FORMS)
def test_a_wait_that_runs_out_is_reported_and_the_handle_keeps_working(form):
    import torch
    from paper_2001_00138_b200 import binding as B
    rows, K, F, skip, plan = FORMS[form]
    got = B.linear_plan(F, K, rows)
    assert {k: got[k] for k in plan} == plan, got
    lin, x, w, y, st = make(F, K, rows)
    want = (x.double() @ w.double().t()).bfloat16()
    lin.run(x, y, rows, stream=st)
    lin.check()
    assert torch.equal(y, want)
    lin.debug_wait(1024, skip)                             # about four milliseconds per wait
    lin.run(x, y, rows, stream=st)
    with pytest.raises(B.PatdnnError) as e:
        lin.check()
    assert e.value.status == E_DEVICE_TIMEOUT
    lin.check()                                            # the report cleared the status word
    lin.debug_wait(0, 0)
    y.fill_(float("nan"))
    lin.run(x, y, rows, stream=st)
    lin.check()
    assert torch.equal(y, want)


def test_the_bound_does_not_count_the_kernel_before():
    """A kernel may arrive while its predecessor runs.  Its waits are for its own copies, so a predecessor that takes longer than they may does
    not use them up: here about 0.06 ms (16 polls), behind a product of several times that."""
    import torch
    rows, K, F = 256, 2 ** 20, 2304
    long, lx, _, ly, st = make(F, K, rows)
    lin, x, w, y, _ = make(128, 64, 3, seed=1)
    lin40, x40, w40, y40, _ = make(128, 64, 40, seed=2)
    long.run(lx, ly, rows, stream=st)
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    a.record()
    long.run(lx, ly, rows, stream=st)
    b.record()
    torch.cuda.synchronize()
    assert a.elapsed_time(b) > 0.4, a.elapsed_time(b)
    for layer in (lin, lin40):
        layer.debug_wait(16, 0)
    from paper_2001_00138_b200 import binding as B
    mx = torch.empty(B.mx4_bytes(40, 64), dtype=torch.uint8, device="cuda")
    B.mx4_quantize(x40, mx, 40, 64, dtype=B.BF16, stream=st)
    for layer, call in ((lin, lambda: lin.run(x, y, 3, stream=st)), (lin40, lambda: lin40.run_mx4(mx, y40, 40, stream=st))):
        long.run(lx, ly, rows, stream=st)
        call()
        layer.check()
    long.check()
    assert torch.equal(y, (x.double() @ w.double().t()).bfloat16())
    assert torch.equal(y40, (x40.double() @ w40.double().t()).bfloat16())


def test_debug_wait_refusals():
    from paper_2001_00138_b200 import binding as B
    lin, *_ = make(32, 32, 1)
    with pytest.raises(B.PatdnnError) as e:
        lin.debug_wait(0, -1)
    assert e.value.status == 2
