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
