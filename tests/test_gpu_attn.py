"""Softmax attention on the GPU against its float64 definition, elementwise
within bounds that count the roundings (mixer_ref)."""

import math

import pytest
import torch

import mixer_ref as R
from paper_2608_09307_amd import linsimp as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def draw(B, H, Hkv, nq, nk, D, dt, seed=0, mag=1.0):
    g = torch.Generator().manual_seed(seed)
    f = lambda *s: (torch.randn(*s, generator=g) * mag).to(dt).to(DEV)  # noqa: E731
    return f(B, H, nq, D), f(B, Hkv, nk, D), f(B, Hkv, nk, D), f(B, H, nq, D)


def lens(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device=DEV)


def train(q, k, v, do, **how):
    out, lse = L.attn_fwd(q, k, v, **how)
    dq, dk, dv = L.attn_bwd(q, k, v, out, lse, do, **how)
    torch.cuda.synchronize()
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


CASES = [
    # B, H, Hkv, nq, nk, D, dtype, causal, window, lens_q, lens_k
    (1, 1, 1, 1, 1, 64, BF, True, 0, None, None),
    (1, 2, 2, 2, 2, 32, BF, True, 0, None, None),
    (2, 3, 1, 33, 33, 64, BF, True, 0, None, None),
    (1, 2, 2, 127, 127, 128, BF, True, 0, None, None),
    (1, 2, 1, 128, 128, 128, BF, False, 0, None, None),
    (1, 8, 8, 129, 129, 64, BF, True, 0, None, None),
    (2, 4, 2, 300, 300, 128, BF, True, 0, None, None),
    (1, 8, 1, 200, 200, 32, BF, True, 0, None, None),
    (1, 2, 2, 257, 257, 64, BF, True, 1, None, None),
    (1, 2, 2, 257, 257, 64, BF, True, 33, None, None),
    (1, 2, 2, 400, 400, 128, BF, True, 64, None, None),
    (1, 2, 2, 400, 400, 128, BF, True, 1000, None, None),
    (4, 2, 1, 190, 190, 64, BF, True, 0, [190, 1, 0, 65], [190, 1, 0, 65]),
    (4, 2, 1, 190, 190, 64, BF, False, 0, [190, 3, 0, 65], [7, 190, 10, 0]),
    (2, 2, 2, 40, 333, 64, BF, True, 0, None, None),
    (2, 2, 2, 40, 333, 128, BF, True, 50, [40, 17], [300, 333]),
    (1, 2, 2, 100, 37, 64, BF, True, 0, None, None),            # more queries than keys: the first rows see none
    (1, 2, 2, 100, 37, 64, BF, False, 0, None, None),
    (2, 1, 1, 5, 1000, 64, BF, True, 0, [5, -3], [1000, 2000]),   # clamped lengths
    (1, 16, 16, 1, 700, 64, BF, True, 0, None, None),
    (1, 2, 2, 1, 1, 32, F32, True, 0, None, None),
    (2, 4, 2, 150, 150, 64, F32, True, 0, None, None),
    (1, 2, 1, 131, 131, 32, F32, False, 0, None, None),
    (3, 2, 1, 200, 200, 32, F32, True, 47, [200, 100, 13], [200, 100, 13]),
    (1, 4, 4, 70, 400, 64, F32, True, 0, None, None),
    (1, 40, 1, 1, 90, 32, F32, True, 0, None, None),              # 40 heads on one key head
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "-".join(map(str, c[:6])) + f"-{str(c[6])[6:]}-{c[7]}-{c[8]}")
def test_forward_and_backward(c):
    B, H, Hkv, nq, nk, D, dt, causal, window, lq, lk = c
    print(f"[attn] {c}", flush=True)
    q, k, v, do = draw(B, H, Hkv, nq, nk, D, dt, seed=nq * 7 + nk)
    got = train(q, k, v, do, causal=causal, window=window, lens_q=lens(lq), lens_k=lens(lk))
    ref = R.attention(q, k, v, do, causal=causal, window=window, lens_q=lq, lens_k=lk)
    for name in got:
        R.within(got[name], ref[name], name)


# ---------------------------------------------------------------------------
# What must not matter
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dt,D", [(BF, 128), (BF, 32), (F32, 64)])
@pytest.mark.parametrize("nq,nk", [(150, 150), (3, 400)])
def test_rows_that_do_not_exist_may_hold_anything(dt, D, nq, nk):
    """Infinities and NaN behind a sequence's lengths leave every result's bits."""
    print(f"[attn] padding {dt} {D} {nq} {nk}", flush=True)
    lq, lk = [nq, nq // 2, 1], [nk, nk - 37, nk // 3]
    clean = draw(3, 4, 2, nq, nk, D, dt, seed=3)
    dirty = [x.clone() for x in clean]
    for b in range(3):
        for x, n in zip(dirty, (lq[b], lk[b], lk[b], lq[b])):
            x[b, :, n:] = math.nan
            x[b, :, n + 1:] = math.inf
    how = dict(lens_q=lens(lq), lens_k=lens(lk))
    got, ref = train(*dirty, **how), train(*clean, **how)
    for name in got:
        assert torch.equal(got[name], ref[name]), name
    assert not got["out"][1, :, lq[1]:].any() and not got["dk"][1, :, lk[1]:].any() and not got["dq"][2, :, 1:].any()


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("window", [1, 31, 32, 40, 64, 65])
def test_mask_edges_inside_a_tile(D, window):
    """Windows and lengths that end in either half of a tile, behind them NaN."""
    print(f"[attn] edges {D} {window}", flush=True)
    lq, lk = [161, 96, 33, 64], [161, 97, 65, 31]
    x = draw(4, 2, 1, 161, 161, D, BF, seed=window)
    ref = R.attention(*x, window=window, lens_q=lq, lens_k=lk)
    for b in range(4):
        for y, n in zip(x, (lq[b], lk[b], lk[b], lq[b])):
            y[b, :, n:] = math.nan
    got = train(*x, window=window, lens_q=lens(lq), lens_k=lens(lk))
    for name in got:
        R.within(got[name], ref[name], name)


@pytest.mark.parametrize("dt,D", [(BF, 128), (BF, 32), (F32, 64)])
@pytest.mark.parametrize("H,Hkv,nq", [(4, 2, 7), (3, 3, 31), (16, 1, 2)])
@pytest.mark.parametrize("window", [0, 1, 33, 300])
def test_a_few_queries(H, Hkv, nq, D, dt, window):
    """Continuations of at most 32 rows per key head, with lengths and a scale of their own."""
    print(f"[attn] few {H} {Hkv} {nq} {D} {dt} {window}", flush=True)
    lq, lk = [nq, nq - 1, 1, 0], [500, 333, 2, 40]
    x = draw(4, H, Hkv, nq, 500, D, dt, seed=window)
    got = train(*x, window=window, scale=0.3, lens_q=lens(lq), lens_k=lens(lk))
    ref = R.attention(*x, window=window, scale=0.3, lens_q=lq, lens_k=lk)
    for name in got:
        R.within(got[name], ref[name], name)


def test_later_keys_do_not_reach_earlier_rows():
    q, k, v, _ = draw(1, 2, 2, 300, 300, 64, BF, seed=5)
    a, la = L.attn_fwd(q, k, v)
    k2, v2 = k.clone(), v.clone()
    k2[:, :, 200:] = 7.0
    v2[:, :, 200:] = -3.0
    b, lb = L.attn_fwd(q, k2, v2)
    assert torch.equal(a[:, :, :200], b[:, :, :200]) and torch.equal(la[:, :, :200], lb[:, :, :200])
    assert not torch.equal(a[:, :, 200:], b[:, :, 200:])


def test_large_scores():
    """Scores in the thousands: one key takes all the weight."""
    q, k, v, do = draw(1, 1, 1, 70, 70, 32, F32, seed=9, mag=1.0)
    q = q * 1000
    got = train(q, k, v, do)
    ref = R.attention(q, k, v, do)
    for name in got:
        R.within(got[name], ref[name], name)


@pytest.mark.parametrize("B,H,Hkv,nq,nk,D,dt", [(1, 2, 1, 64, 4000, 64, BF), (2, 8, 2, 700, 700, 128, BF),
                                              (1, 6, 1, 333, 333, 32, F32), (1, 32, 2, 1, 9000, 128, BF)])
def test_runs_are_the_same_bits(B, H, Hkv, nq, nk, D, dt):
    x = draw(B, H, Hkv, nq, nk, D, dt, seed=1)
    a = train(*x)
    for _ in range(3):
        b = train(*x)
        for name in a:
            assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("B,H,Hkv,nq,nk,D,dt,window", [
    (1, 2, 1, 64, 4000, 64, BF, 0), (1, 4, 1, 20, 3000, 128, BF, 0), (1, 2, 2, 256, 2500, 32, BF, 700),
    (1, 8, 1, 1000, 1000, 64, BF, 0), (1, 4, 4, 1, 5000, 32, F32, 0), (2, 6, 1, 300, 300, 64, F32, 0)])
def test_sweeps_in_pieces(B, H, Hkv, nq, nk, D, dt, window):
    """Few workgroups over a long axis: the keys (the queries) split and joined."""
    print(f"[attn] pieces {B, H, Hkv, nq, nk, D, dt, window}", flush=True)
    x = draw(B, H, Hkv, nq, nk, D, dt, seed=2)
    got, ref = train(*x, window=window), R.attention(*x, window=window)
    for name in got:
        R.within(got[name], ref[name], name)


def test_gradients_against_differences():
    """Central differences of sum(do * out) along random directions, float32: the
    step h moves the sum by h d, with an error of h^2 from the third derivative
    and of a few 1e-7 |sum of terms| / h from rounding: 2e-3 at h = 2e-2."""
    q, k, v, do = draw(1, 2, 1, 40, 40, 32, F32, seed=11, mag=0.5)
    got = train(q, k, v, do)
    g = torch.Generator().manual_seed(1)
    for i, name in enumerate(("dq", "dk", "dv")):
        x = [q, k, v]
        dirn = torch.randn(x[i].shape, generator=g).to(DEV)
        dirn /= dirn.norm()
        f = []
        for sgn in (1, -1):
            y = list(x)
            y[i] = x[i] + sgn * 2e-2 * dirn
            f.append((L.attn_fwd(*y)[0].double() * do.double()).sum().item())
        num, ana = (f[0] - f[1]) / 4e-2, (got[name].double() * dirn.double()).sum().item()
        assert abs(num - ana) <= 2e-3 * max(1.0, abs(ana)), (name, num, ana)


# ---------------------------------------------------------------------------
# The single-token step
# ---------------------------------------------------------------------------

def step_ref(kc, vc, pos, q, k, v):
    """The step's caches and, by the attention of the tokens in the ring, its out."""
    kc, vc = kc.clone(), vc.clone()
    B, Hkv, cap, D = kc.shape
    outs = []
    for b, p in enumerate(pos):
        if p < 0:
            outs.append((torch.zeros(q.shape[1], D, dtype=torch.float64), torch.full((q.shape[1], D), 1e-30, dtype=torch.float64)))
            continue
        kc[b, :, p % cap], vc[b, :, p % cap] = k[b], v[b]
        m = min(p + 1, cap)
        o, bound = R.attention(q[b:b + 1, :, None], kc[b:b + 1, :, :m], vc[b:b + 1, :, :m], causal=False)["out"]
        outs.append((o[0, :, 0], bound[0, :, 0]))
    return kc, vc, (torch.stack([o for o, _ in outs]), torch.stack([x for _, x in outs]))


@pytest.mark.parametrize("H,Hkv,cap,D,dt,pos", [
    (2, 2, 1, 64, BF, [0, 5, 1 << 40]), (4, 2, 7, 32, BF, [0, 6, 7, 13]), (6, 6, 100, 64, BF, [0, 31, 32, 99, 100, 250]),
    (16, 4, 500, 128, BF, [3, 498, 499, 500, 777]), (40, 1, 65, 32, BF, [0, 64, 1000]), (8, 1, 3000, 128, BF, [2999, 10]),
    (4, 2, 90, 64, F32, [0, 40, 89, 95]), (2, 1, 33, 32, F32, [32, -1, 33, (1 << 63) - 1]), (4, 4, 40, 128, BF, [-1, -7]),
    (70, 2, 50, 64, BF, [49, 20]),
])
def test_step(H, Hkv, cap, D, dt, pos):
    print(f"[attn] step {H, Hkv, cap, D, dt, pos}", flush=True)
    B = len(pos)
    q, kc, vc, _ = draw(B, H, Hkv, 1, cap, D, dt, seed=cap)
    _, k, v, _ = draw(B, H, Hkv, 1, 1, D, dt, seed=cap + 1)
    q, k, v = q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), v[:, :, 0].contiguous()
    for b, p in enumerate(pos):                               # slots no token has reached
        if 0 <= p < cap:
            kc[b, :, p:], vc[b, :, p:] = math.nan, math.inf
    rk, rv, ref = step_ref(kc, vc, pos, q, k, v)
    p = torch.tensor(pos, dtype=torch.int64, device=DEV)
    out = L.attn_step(kc, vc, p, q, k, v)
    torch.cuda.synchronize()
    assert p.tolist() == pos
    bits = lambda x: x.view(torch.int16 if dt == BF else torch.int32)  # noqa: E731  (unused slots hold NaN)
    assert torch.equal(bits(kc), bits(rk)) and torch.equal(bits(vc), bits(rv))
    R.within(out, ref, "out")


def test_steps_follow_the_prompt():
    """A padded batch of prompts through the forward, its keys in the cache, then
    tokens one at a time: the rows of one forward over everything."""
    B, H, Hkv, D, n, cap = 3, 4, 2, 64, 40, 64
    first = [40, 17, 29]
    q, k, v, _ = draw(B, H, Hkv, cap, cap, D, BF, seed=21)
    whole, _ = L.attn_fwd(q, k, v)
    kc, vc = torch.full_like(k, math.nan), torch.full_like(v, math.nan)
    for b, m in enumerate(first):
        kc[b, :, :m], vc[b, :, :m] = k[b, :, :m], v[b, :, :m]
    out, _ = L.attn_fwd(q[:, :, :n].contiguous(), kc, vc, lens_q=lens(first), lens_k=lens(first))
    for b, m in enumerate(first):
        d = (out[b, :, :m].float() - whole[b, :, :m].float()).abs()
        assert d.max() <= 2 ** -7 * whole[b].abs().max()        # (both are within 2^-8 of the same value's terms)
    pos = torch.tensor(first, dtype=torch.int64, device=DEV)
    for _ in range(20):
        at = pos.tolist()
        tok = [torch.stack([x[b, :, at[b]] for b in range(B)]).contiguous() for x in (q, k, v)]
        o = L.attn_step(kc, vc, pos, *tok)
        for b in range(B):
            d = (o[b].float() - whole[b, :, at[b]].float()).abs()
            assert d.max() <= 2 ** -7 * whole[b].abs().max(), (b, at)
        pos += 1


def test_step_past_32_bits():
    """Caches of more than 2^32 elements: the second sequence's slots lie behind them."""
    cap, D = (1 << 25) + 3, 128
    kc = torch.empty(2, 1, cap, D, dtype=BF, device=DEV)
    vc = torch.empty_like(kc)
    x, k0, v0, _ = draw(1, 2, 1, 100, 200, D, BF, seed=4)
    kc[1, :, :200], vc[1, :, :200] = k0[0], v0[0]
    q, k, v = x[:, :, 0], k0[:, :, 199], v0[:, :, 199]
    both = [torch.cat([y, y]).contiguous() for y in (q, k, v)]
    out = L.attn_step(kc, vc, torch.tensor([0, 199], device=DEV), *both)
    ref = R.attention(q[:, :, None], k0, v0, causal=False)["out"]
    R.within(out[1:, :, None], ref, "out")
    assert torch.equal(out[0].float(), v[0].float().expand(2, D))            # one token: its value
    lk = lens([1, 200])
    o2, _ = L.attn_fwd(both[0][:, :, None].contiguous(), kc, vc, lens_q=lens([1, 1]), lens_k=lk)
    R.within(o2[1:], ref, "out")


# ---------------------------------------------------------------------------
# Graphs and streams
# ---------------------------------------------------------------------------

def test_captured_calls_replay():
    x = draw(1, 4, 2, 200, 1000, 64, BF, seed=6)
    d = L.attn_dims(x[0], x[1])
    ws = L.alloc_bytes(L.attn_workspace_size(d, True), x[0].device)
    kc, vc = x[1].clone(), x[2].clone()
    tok = [y[:, :, 0].contiguous() for y in (x[0], x[1], x[2])]
    pos = torch.tensor([500], device=DEV)
    out, lse, grads = torch.empty_like(x[0]), torch.empty(1, 4, 200, device=DEV), [torch.empty_like(y) for y in x[:3]]
    so = torch.empty_like(tok[0])

    def calls():
        L.attn_fwd(*x[:3], out=out, lse=lse, workspace=ws)
        L.attn_bwd(*x[:3], out, lse, x[3], grads=grads, workspace=ws)
        L.attn_step(kc, vc, pos, *tok, out=so, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        calls()
    for seed in (31, 32, 33):
        y = draw(1, 4, 2, 200, 1000, 64, BF, seed=seed)
        for a, b in zip(x, y):
            a.copy_(b)
        pos.fill_(seed)
        g.replay()
        torch.cuda.synchronize()
        got = [z.clone() for z in (out, lse, *grads, so)]
        calls()                                               # the same, eagerly
        torch.cuda.synchronize()
        for a, b in zip(got, (out, lse, *grads, so)):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    xs = [draw(1, 4, 2, 500, 500, 64, BF, seed=s) for s in (41, 42)]
    ref = [train(*x) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                o, z = L.attn_fwd(*x[:3])
                got.append((o, z, *L.attn_bwd(*x[:3], o, z, x[3])))
        torch.cuda.synchronize()
        for a, b in zip(got, ref):
            for y, z in zip(a, b.values()):
                assert torch.equal(y, z)
