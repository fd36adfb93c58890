"""The gated linear recurrence on the GPU against its float64 definition, row by
row, elementwise within bounds that count the roundings (mixer_ref)."""

import math

import pytest
import torch

import mixer_ref as R
from paper_2608_09307_amd import linsimp as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def gates(kind, shape, gen):
    x = torch.randn(shape, generator=gen)
    if kind == "slow":
        return torch.nn.functional.logsigmoid(x) / 16
    if kind == "none":
        return torch.zeros(shape)
    if kind == "strong":                                      # every row forgets almost all
        return -10.0 - x.abs()
    rate = torch.exp(-math.log(4096.0) * torch.rand(shape[-1], generator=gen))
    g = -rate * torch.exp(0.5 * x)
    if kind == "reset":
        g = torch.where(torch.rand(shape, generator=gen) < 1 / 64, torch.full_like(g, -40.0), g)
    if kind == "clear":                                       # cleared channels, some in rows next to each other
        g = torch.where(torch.rand(shape, generator=gen) < 1 / 16, torch.full_like(g, -math.inf), g)
    return g


def draw(B, H, n, D, dt, kind, state, seed=0):
    gen = torch.Generator().manual_seed(seed)
    f = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x = {nm: f(B, H, n, D) for nm in ("q", "k", "v", "dout")}
    x["k"] *= D ** -0.5
    x["g"] = gates(kind, (B, H, n, D), gen)
    x = {nm: y.to(dt).to(DEV) for nm, y in x.items()}
    for nm in ("s0", "ds1"):
        x[nm] = f(B, H, D, D).to(DEV) if state else None
    return x


def train(x, lens=None, scale=None):
    a = (x["q"], x["k"], x["v"], x["g"])
    out, s1 = L.glr_fwd(*a, s0=x["s0"], lens=lens, scale=scale)
    dq, dk, dv, dg, ds0 = L.glr_bwd(*a, x["dout"], s0=x["s0"], lens=lens, ds1=x["ds1"], scale=scale, want_ds0=True)
    torch.cuda.synchronize()
    return {"out": out, "s1": s1, "dq": dq, "dk": dk, "dv": dv, "dg": dg, "ds0": ds0}


CASES = [
    # B, H, n, D, dtype, gates, state, lens
    (1, 1, 1, 32, BF, "slow", False, None),
    (1, 1, 1, 32, BF, "slow", True, None),
    (1, 1, 2, 64, BF, "slow", False, None),
    (1, 2, 31, 64, BF, "mixed", True, None),
    (2, 1, 32, 128, BF, "mixed", True, None),
    (1, 2, 33, 32, BF, "mixed", False, None),
    (1, 1, 64, 128, BF, "slow", False, None),
    (1, 2, 100, 64, BF, "mixed", True, None),
    (1, 1, 300, 128, BF, "mixed", True, None),
    (1, 1, 333, 64, BF, "none", True, None),
    (1, 1, 100, 64, BF, "strong", True, None),
    (1, 2, 200, 64, BF, "reset", True, None),
    (1, 1, 130, 128, BF, "reset", False, None),
    (1, 1, 97, 32, BF, "clear", True, None),
    (1, 1, 70, 128, BF, "clear", True, None),
    (4, 1, 90, 64, BF, "mixed", True, [90, 0, 33, 64]),
    (3, 2, 140, 128, BF, "reset", True, [1, 200, -4]),
    (1, 1, 1000, 32, BF, "mixed", True, None),
    (1, 1, 1, 32, F32, "mixed", True, None),
    (1, 2, 100, 64, F32, "mixed", True, None),
    (2, 1, 65, 32, F32, "reset", True, None),
    (1, 1, 97, 64, F32, "clear", True, None),
    (3, 1, 200, 32, F32, "slow", False, [200, 31, 100]),
    (1, 1, 64, 64, F32, "strong", False, None),
    (1, 1, 700, 32, F32, "mixed", True, None),
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(map(str, c[:4])) + f"-{str(c[4])[6:]}-{c[5]}-{c[6]}")
def test_forward_and_backward(c):
    B, H, n, D, dt, kind, state, lens = c
    print(f"[glr] {c}", flush=True)
    x = draw(B, H, n, D, dt, kind, state, seed=n + D)
    got = train(x, None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV))
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], x["dout"], x["s0"], x["ds1"], lens)
    for name in got:
        R.within(got[name], ref[name], name)


@pytest.mark.parametrize("D,dt", [(32, BF), (64, BF), (128, BF), (32, F32), (64, F32)])
def test_steps_equal_the_rows(D, dt):
    B, H, n = 2, 3, 40
    x = draw(B, H, n, D, dt, "mixed", True, seed=D)
    state = x["s0"].clone()
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], s0=x["s0"])
    rows = [L.glr_step(state, *(x[nm][:, :, t].contiguous() for nm in "qkvg")) for t in range(n)]
    torch.cuda.synchronize()
    R.within(torch.stack(rows, 2), ref["out"], "out")
    R.within(state, ref["s1"], "state")
