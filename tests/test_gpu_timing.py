"""The library's own kernel timing over the mixers: every launch has its two events
and is counted under a name of its own."""

import pytest
import torch

from test_gpu_glr import BF, F32, draw, train
from paper_2608_09307_amd import linsimp as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt,state", [(BF, False), (BF, True), (F32, True)])
def test_both_ways_of_the_recurrence_are_counted(dt, state):
    """A segment is taken the short way, and again the exact way where that gave up:
    two launches, with different times."""
    x = draw(1, 2, 200, 32, dt, "clear", state)
    a = [x[nm] for nm in "qkvg"]
    train(x)
    L.timing_enable(True)
    try:
        L.timing_read()
        for _ in range(3):
            L.glr_fwd(*a, s0=x["s0"], want_state=state)
            L.glr_bwd(*a, x["dout"], s0=x["s0"], ds1=x["ds1"], want_ds0=state)
        torch.cuda.synchronize()
        got = L.timing_read()
    finally:
        L.timing_enable(False)
    for name in ("glr_fwd", "glr_fwd_exact", "glr_bwd", "glr_bwd_exact"):
        assert name in got, got
        assert got[name][1] == 3 and got[name][0] > 0, got
