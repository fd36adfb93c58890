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


# ---------------------------------------------------------------------------
# What must not matter
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dt,D,kind", [(BF, 128, "mixed"), (BF, 64, "reset"), (F32, 32, "mixed")])
def test_rows_that_do_not_exist_may_hold_anything(dt, D, kind):
    print(f"[glr] padding {dt} {D} {kind}", flush=True)
    ln = [150, 70, 0, 33]
    x = draw(4, 2, 150, D, dt, kind, True, seed=3)
    dirty = {nm: None if y is None else y.clone() for nm, y in x.items()}
    for nm in ("q", "k", "v", "g", "dout"):
        for b, m in enumerate(ln):
            dirty[nm][b, :, m:] = math.nan
            dirty[nm][b, :, m + 1:] = math.inf
    t = torch.tensor(ln, dtype=torch.int32, device=DEV)
    got, ref = train(dirty, t), train(x, t)
    for name in got:
        assert torch.equal(got[name], ref[name]), name
    assert not got["out"][1, :, 70:].any() and not got["dg"][2].any()
    assert torch.equal(got["s1"][2], x["s0"][2]) and torch.equal(got["ds0"][2], x["ds1"][2])


@pytest.mark.parametrize("D,dt,kind", [(64, BF, "mixed"), (128, BF, "reset"), (32, F32, "slow")])
def test_a_sequence_in_two_calls(D, dt, kind):
    """The state handed from one call to the next, in place of it where the header
    allows that, against the whole sequence."""
    B, H, n, cut = 2, 2, 200, 77
    x = draw(B, H, n, D, dt, kind, True, seed=8)
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], s0=x["s0"])
    state = x["s0"].clone()
    outs = []
    for a, b in ((0, cut), (cut, n)):
        o, s = L.glr_fwd(*(x[nm][:, :, a:b].contiguous() for nm in "qkvg"), s0=state, s1=state)
        assert s is state
        outs.append(o)
    torch.cuda.synchronize()
    R.within(torch.cat(outs, 2), ref["out"], "out")
    R.within(state, (ref["s1"][0], 2 * ref["s1"][1]), "state")


@pytest.mark.parametrize("B,H,n,D,dt,kind", [(1, 1, 3000, 64, BF, "mixed"), (1, 2, 2500, 32, F32, "mixed"),
                                          (1, 1, 1500, 128, BF, "reset")])
def test_long_sequences_in_segments(B, H, n, D, dt, kind):
    print(f"[glr] long {B, H, n, D, dt, kind}", flush=True)
    x = draw(B, H, n, D, dt, kind, True, seed=n)
    got = train(x)
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], x["dout"], x["s0"], x["ds1"])
    for name in got:
        R.within(got[name], ref[name], name)


@pytest.mark.parametrize("scale", [0.0, -0.5, 3.0])
def test_scales(scale):
    x = draw(1, 2, 70, 32, F32, "mixed", True, seed=5)
    got = train(x, scale=scale)
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], x["dout"], x["s0"], x["ds1"], scale=scale)
    for name in got:
        R.within(got[name], ref[name], name)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("mag", [1.0, 2.0 ** 15])
@pytest.mark.parametrize("gate", [-2.55, -2.65, -30.0])
def test_decays_at_the_limit_of_the_short_way(gate, mag, dt):
    """16 rows of -2.55 decay by 2^58.9, of -2.65 by 2^61.2 (the limit is 2^60), with
    values that have to fit beside such factors."""
    print(f"[glr] limit {gate} {mag} {dt}", flush=True)
    x = draw(2, 1, 100, 64, dt, "none", True, seed=21)
    x["g"] += gate
    for nm in ("q", "k", "v", "dout"):
        x[nm] *= mag
    got = train(x)
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], x["dout"], x["s0"], x["ds1"])
    for name in got:
        R.within(got[name], ref[name], name)


def test_growing_gates():
    """g above zero is an ordinary exponential (the state grows)."""
    x = draw(1, 1, 64, 32, F32, "none", True, seed=5)
    x["g"] += 0.05
    got = train(x)
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], x["dout"], x["s0"], x["ds1"])
    for name in got:
        R.within(got[name], ref[name], name)


def test_one_chunk_in_a_long_sequence_takes_the_exact_way():
    x = draw(1, 2, 600, 64, BF, "slow", True, seed=6)
    x["g"][0, 0, 300:303, 5] = -math.inf
    x["g"][0, 1, 10, :] = -200.0
    got = train(x)
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], x["dout"], x["s0"], x["ds1"])
    for name in got:
        R.within(got[name], ref[name], name)


@pytest.mark.parametrize("B,H,n,D,dt,kind", [(2, 3, 700, 64, BF, "mixed"), (1, 2, 300, 128, BF, "reset"),
                                          (1, 2, 300, 32, F32, "mixed")])
def test_runs_are_the_same_bits(B, H, n, D, dt, kind):
    x = draw(B, H, n, D, dt, kind, True, seed=1)
    a = train(x)
    for _ in range(3):
        b = train(x)
        for name in a:
            assert torch.equal(a[name], b[name]), name


def test_gradients_against_differences():
    """Central differences along random directions (see the attention's test)."""
    x = draw(1, 2, 50, 32, F32, "mixed", True, seed=12)
    got = train(x)

    def value(y):
        out, s1 = L.glr_fwd(y["q"], y["k"], y["v"], y["g"], s0=y["s0"])
        return (out.double() * x["dout"].double()).sum().item() + (s1.double() * x["ds1"].double()).sum().item()

    gen = torch.Generator().manual_seed(1)
    for nm in ("q", "k", "v", "g", "s0"):
        dirn = torch.randn(x[nm].shape, generator=gen).to(DEV)
        dirn /= dirn.norm()
        h = 2e-2
        num = (value({**x, nm: x[nm] + h * dirn}) - value({**x, nm: x[nm] - h * dirn})) / (2 * h)
        ana = (got["d" + nm].double() * dirn.double()).sum().item()
        assert abs(num - ana) <= 5e-3 * max(1.0, abs(ana)), (nm, num, ana)


def test_captured_calls_replay():
    x = draw(1, 3, 500, 64, BF, "mixed", True, seed=2)
    a = [x[nm] for nm in "qkvg"]
    ws = L.alloc_bytes(L.glr_workspace_size(L.glr_dims(x["q"]), True), x["q"].device)
    out, s1 = torch.empty_like(x["q"]), torch.empty_like(x["s0"])
    grads = [torch.empty_like(y) for y in a]
    state = x["s0"].clone()
    tok = [y[:, :, 0].contiguous() for y in a]
    so = torch.empty_like(tok[0])

    def calls():
        L.glr_fwd(*a, s0=x["s0"], out=out, s1=s1, workspace=ws)
        L.glr_bwd(*a, x["dout"], s0=x["s0"], ds1=x["ds1"], grads=grads, want_ds0=False, workspace=ws)
        state.copy_(s1)
        L.glr_step(state, *tok, out=so)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for seed, kind in ((31, "mixed"), (32, "reset"), (33, "slow")):
        y = draw(1, 3, 500, 64, BF, kind, True, seed=seed)
        for nm in x:
            x[nm].copy_(y[nm])
        g.replay()
        torch.cuda.synchronize()
        got = [z.clone() for z in (out, s1, *grads, state, so)]
        calls()
        torch.cuda.synchronize()
        for u, v in zip(got, (out, s1, *grads, state, so)):
            assert torch.equal(u, v)


def test_two_streams_at_once():
    xs = [draw(1, 4, 600, 64, BF, kind, False, seed=s) for s, kind in ((41, "mixed"), (42, "reset"))]
    ref = [train(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                a = [x[nm] for nm in "qkvg"]
                o, s1 = L.glr_fwd(*a)
                got.append((o, s1, *L.glr_bwd(*a, x["dout"], want_ds0=True)))
        torch.cuda.synchronize()
        for y, z in zip(got, ref):
            for u, v in zip(y, z.values()):
                assert torch.equal(u, v)
