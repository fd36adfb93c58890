"""What independent roundings may do to the gated linear recurrence, block by block.

mixer_ref bounds every element by the worst case, a sum of absolute values over a
D x D state, which a value of the size of the result can hide in.  Here the
roundings are counted as what they are for inputs of random sign: independent, each
with a standard deviation of at most u / sqrt(3) of the term it rounds (u the unit
roundoff of the operand type; a rounding is uniform within half a step).

A result is a sum over elementary terms, for dg_r
    scale k_sd v_se q_td do_te decay(s .. t)_d     over s < r <= t and e
(with s0 or ds1 in the place of k v or q do), and every factor of a term, every
partial sum it enters as an operand and the store round it at most N times:
    out   q, k, the pair weight or the state, the store                     N = 4
    dq    k, the pair weight or the state, the store                        N = 3
    dk    q, the pair weight or the gradient's state, the store             N = 3
    dv    q, k, the pair weight or the gradient's state, the store          N = 4
    dg    q, k, both states (or the pair weight and one state), the store   N = 5
Partial sums of random terms have the mean square of the sum of the terms' squares,
V, so an element's error has a variance of at most N u^2 / 3 V, and V follows the
recurrence itself with every input squared and the decays doubled.  Rows whose pairs
cancel in dg's sums over later rows add float32 rounding: 64 e (e = 2^-24: up to 32
rows of a sum, a product and a conversion each) of the root of C, the squares of
what is summed there.

Over a block of 32 rows of one head the squared errors add up; errors that several
rows share (W, a state) leave fewer independent ones, so three standard deviations
are allowed on the block's root mean square.
"""

import torch

import mixer_ref as R

E32 = 2.0 ** -24
ROUNDINGS = {"out": 4, "dq": 3, "dk": 3, "dv": 4, "dg": 5}
ROWS = 32


def _blocks(x):
    """[B, H, n, D] -> sums over blocks of 32 rows and all channels, [B, H, blocks]."""
    B, H, n, D = x.shape
    pad = -n % ROWS
    return torch.nn.functional.pad(x, (0, 0, 0, pad)).view(B, H, -1, ROWS * D).sum(-1)


def squares(x, lens=None, scale=None):
    """V of out, dq, dk, dv, dg and C of dg, from the inputs' squares."""
    D = x["q"].shape[-1]
    scale = D ** -0.5 if scale is None else scale
    sq = {nm: None if y is None else y.detach().cpu().double() ** 2 for nm, y in x.items() if nm != "g"}
    g2 = 2 * x["g"].detach().cpu().double()
    got = R.recurrence(sq["q"], sq["k"], sq["v"], g2, sq["dout"], sq["s0"], sq["ds1"], lens, scale ** 2)
    V = {nm: got[nm][0] for nm in ROUNDINGS}
    n = g2.shape[2]
    c = sq["q"] * V["dq"] + sq["k"] * V["dk"]
    if lens is not None:
        for b, m in enumerate(lens):
            c[b, :, min(max(m, 0), n):] = 0
    # sums of later rows inside a chunk, and what passes its end (W: of the size of dg there)
    tail = torch.zeros_like(c)
    for t0 in range(0, n, ROWS):
        part = c[:, :, t0:t0 + ROWS]
        tail[:, :, t0:t0 + ROWS] = part.flip(2).cumsum(2).flip(2) + V["dg"][:, :, t0:t0 + ROWS].amax(2, keepdim=True)
    return V, tail


def block_bounds(x, lens=None, scale=None, deviations=3.0):
    """{name: [B, H, blocks]} bounds on the root of the summed squares of the errors."""
    u = R.unit(x["q"].dtype)
    V, C = squares(x, lens, scale)
    b = {nm: deviations ** 2 * ROUNDINGS[nm] * u * u / 3 * _blocks(V[nm]) for nm in ROUNDINGS}
    b["dg"] = b["dg"] + (64 * E32) ** 2 * _blocks(C)
    # three figures of float32 sums in the others (a value of few terms may be exact)
    return {nm: (y + (8 * E32) ** 2 * _blocks(V[nm])).sqrt() + 1e-30 for nm, y in b.items()}


def block_errors(got, val):
    return _blocks((got.detach().cpu().double() - val) ** 2).sqrt()


def within_blocks(got, val, bound, name):
    worst = (block_errors(got, val) / bound).max().item()
    assert worst <= 1.0, f"{name}: a block is off by {worst:.3g} times its bound"
    return worst


def dg_parts(x, scale=None):
    """dg by where its terms come from, {(source, sink): [B, H, n, D]}: a source is the
    state s0, an earlier chunk or the row's own chunk, a sink the row's own chunk, a
    later one or ds1."""
    f = {nm: None if y is None else y.detach().cpu().double() for nm, y in x.items()}
    B, H, n, D = f["q"].shape
    scale = D ** -0.5 if scale is None else scale
    a = f["g"].exp()
    zero = torch.zeros(B, H, D, D, dtype=torch.float64)
    S = {"s0": zero if f["s0"] is None else f["s0"], "earlier": zero, "own": zero}
    before = []
    for t in range(n):
        if t % ROWS == 0:
            S = {"s0": S["s0"], "earlier": S["earlier"] + S["own"], "own": zero}
        S = {nm: s * a[:, :, t, :, None] for nm, s in S.items()}
        before.append(S)
        S = {**S, "own": S["own"] + f["k"][:, :, t, :, None] * f["v"][:, :, t, None]}
    T = {"ds1": zero if f["ds1"] is None else f["ds1"], "later": zero, "own": zero}
    parts = {(s, t): torch.zeros(B, H, n, D, dtype=torch.float64) for s in S for t in T}
    for t in range(n - 1, -1, -1):
        if t % ROWS == ROWS - 1 or t == n - 1:
            T = {"ds1": T["ds1"], "later": T["later"] + T["own"], "own": zero}
        T = {**T, "own": T["own"] + scale * f["q"][:, :, t, :, None] * f["dout"][:, :, t, None]}
        for s in S:
            for r in T:
                parts[s, r][:, :, t] = (T[r] * before[t][s]).sum(3)
        T = {nm: y * a[:, :, t, :, None] for nm, y in T.items()}
    return parts
