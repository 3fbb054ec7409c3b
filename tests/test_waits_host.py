"""Bounded waits whose outcome decides what a warp does next.  The instructions behind them (reads of tensor memory, cluster barriers) are executed
by whole warps, so the lanes of a warp have to agree: one that gave up must not leave the others.  Shown in the source, without a device."""
import os
import re

import pytest

from paper_2001_00138_b200 import build


@pytest.mark.parametrize("name", ["gated.cu", "mx8_linear.cu", "mx4_linear.cu"])
def test_lanes_of_a_warp_agree_on_a_wait(name):
    """Every role of these kernels is a whole warp: only warp_wait's outcome (a vote) may be used, that of a lane's own wait not."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, name)).read())
    used = [m.group(0) for m in re.finditer(r"[^\n]*(?:!|=|&&|\|\||\bif \(|\breturn\b)\s*mbar_wait\([^\n]*", text)]
    assert "warp_wait(" in text and not used, used


def loops(text):
    """(head, body) of every for loop with braces."""
    for m in re.finditer(r"\bfor \(", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        if text[at:at + 2] != " {":
            continue
        begin = at + 2
        depth, at = 1, begin
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield text[m.start():begin], text[begin:at]


@pytest.mark.parametrize("name", ["umma_conv.cu", "umma_chain.cu"])
def test_nobody_leaves_a_loop_whose_turns_meet_at_a_barrier(name):
    """Warps that meet at a named barrier (which has no bound) once per turn: one that gave up on a wait keeps meeting it and skips the work."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, name)).read())
    found = 0
    for head, body in loops(text):
        inner = body
        for h, b in loops(body):                           # (what a loop inside leaves is its own)
            if "bar.sync" not in b:
                inner = inner.replace(b, "")
        if "bar.sync" in inner:
            found += 1
            assert "break;" not in inner, head
    assert found >= 1 or name == "umma_chain.cu"


def test_whole_warps_read_tensor_memory_in_the_convolutions():
    """Behind the epilogue's waits (for a finished accumulator: bar_acc, bar_af) come warp-wide reads of tensor memory."""
    for name in ("umma_conv.cu", "umma_chain.cu"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, name)).read())
        for m in re.finditer(r"mbar_wait\(bar_(?:acc|af)\b", text):
            around = text[max(0, m.start() - 40):m.end() + 140]
            assert "__all_sync(" in around or "__any_sync(" in around, (name, around)


def test_waits_of_no_handle():
    from paper_2001_00138_b200 import binding as B
    lib = B.load()
    for call in (lib.patdnn_rms_check, lib.patdnn_linear8_check, lib.patdnn_gated_check):
        assert call(None) == 1                             # E_NULL
    for call in (lib.patdnn_rms_debug_wait, lib.patdnn_linear8_debug_wait, lib.patdnn_gated_debug_wait):
        assert call(None, 1024, 1) == 1
