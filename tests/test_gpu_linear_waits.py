"""Bounded waits of the linear layer's kernels: one that runs out ends the kernel through its normal exit, patdnn_linear_check reports it, and the
handle works again afterwards.

Nothing here faults, traps or hangs the GPU: the bound is shortened to about a millisecond and the copies of one column tile are left out
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
    lin.debug_wait(1024, skip)                             # about a millisecond per wait
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


def test_debug_wait_refusals():
    from paper_2001_00138_b200 import binding as B
    lin, *_ = make(32, 32, 1)
    with pytest.raises(B.PatdnnError) as e:
        lin.debug_wait(0, -1)
    assert e.value.status == 2
