"""Bounded waits of the gated block's kernel that reads weights as they lie (rows that are not whole 16-byte units apart), alone and in clusters; the other
forms are in test_gpu_gated."""
import pytest

from test_gpu_gated import Case, E_DEVICE_TIMEOUT

pytestmark = pytest.mark.gpu
FORMS = {  # rows, K, F, what weights' rows are further apart than they are long, block that is left out, what patdnn_gated_plan_strided says
    "eight phases, one range": (3, 1001, 9000, 0, 2, dict(splits=1, few_rows=1)),
    "eight phases, first block": (3, 1001, 9000, 0, 1, dict(splits=1, few_rows=1)),
    "eight phases, cluster of two": (8, 4099, 3500, 0, 3, dict(splits=2, few_rows=1)),
    "four phases, cluster of four": (5, 4098, 1700, 0, 1, dict(splits=4, few_rows=1)),
    "two phases, cluster of eight": (40, 4100, 330, 0, 2, dict(splits=8, few_rows=1)),
}


@pytest.mark.parametrize("form", FORMS)
def test_a_wait_that_runs_out_is_reported_and_the_handle_keeps_working(form):
    """The bound is shortened to a few milliseconds and the copies of one block are left out, so that the consumers' wait for them runs out."""
    import torch
    from paper_2001_00138_b200 import binding as B
    M, K, F, wslack, skip, plan = FORMS[form]
    got = B.gated_plan(F, K, M, 0, K + wslack)
    assert {k: got[k] for k in plan} == plan and (K + wslack) % 8, got
    c = Case(M, K, F, "bf16", "silu", False, wslack=wslack)
    c.forward()
    want, gu = c.h.clone(), c.gu.clone()
    c.block.debug_wait(1024, skip)
    with pytest.raises(B.PatdnnError) as e:
        c.forward()
    assert e.value.status == E_DEVICE_TIMEOUT
    c.block.check()                                        # the report cleared the status word
    c.block.debug_wait(0, 0)
    c.h.fill_(float("nan"))
    c.gu.fill_(float("nan"))
    c.forward()
    assert torch.equal(c.h, want) and torch.equal(c.gu, gu)
