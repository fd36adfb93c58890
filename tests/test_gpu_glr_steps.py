"""The recurrence's single-token step with gates that clear channels, against the
definition and against the forward of one row."""

import math

import pytest
import torch

import mixer_ref as R
from test_gpu_glr import BF, DEV, F32, draw
from paper_2608_09307_amd import linsimp as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,dt", [(32, BF), (64, BF), (128, BF), (32, F32), (64, F32)])
@pytest.mark.parametrize("kind", ["clear", "reset", "strong", "none"])
def test_gates_of_a_step(D, dt, kind):
    print(f"[glr] step {D} {dt} {kind}", flush=True)
    n = 24
    x = draw(2, 3, n, D, dt, kind, True, seed=D)
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], s0=x["s0"])
    state = x["s0"].clone()
    rows = [L.glr_step(state, *(x[nm][:, :, t].contiguous() for nm in "qkvg")) for t in range(n)]
    torch.cuda.synchronize()
    R.within(torch.stack(rows, 2), ref["out"], "out")
    R.within(state, ref["s1"], "state")


@pytest.mark.parametrize("D,dt", [(128, BF), (64, F32)])
def test_a_cleared_channel_keeps_the_token_alone(D, dt):
    """exp(-inf) = 0 whatever finite state it meets, in the step and in a forward of one row."""
    x = draw(1, 2, 1, D, dt, "slow", True, seed=9)
    x["g"][:, :, :, ::3] = -math.inf
    x["s0"] *= 2.0 ** 40
    tok = [x[nm][:, :, 0].contiguous() for nm in "qkvg"]
    state = x["s0"].clone()
    L.glr_step(state, *tok)
    _, s1 = L.glr_fwd(*(x[nm] for nm in "qkvg"), s0=x["s0"])
    torch.cuda.synchronize()
    kv = tok[1].float()[..., None] * tok[2].float()[..., None, :]
    assert torch.equal(state[:, :, ::3], kv[:, :, ::3])
    d = (s1[:, :, ::3] - kv[:, :, ::3]).abs()
    assert (d <= 2.0 ** -16 * kv[:, :, ::3].abs() + 1e-30).all()       # (rows of two terms: 2^-17)
