"""Softmax attention and the gated linear recurrence from their definitions, in
float64 on the CPU, with elementwise bounds on what a kernel's roundings may
change.

Bounds count worst cases.  With u the unit roundoff of the stored type (bf16
2^-8, float32 2^-24) and e = 2^-24 for every float32 operation:
  recurrence  a pair's weight is a product of scaled rows, each rounded to the operand
              type (u), of a rounded pair weight or state (u) and of float32 decays (whose
              errors, with those of the float32 sums, are counted 4 n + 200 times e);
              float32 states of bf16 inputs are sums of two-term rows (u^2)
  attention   a score is off by (D + 4) e sum_d |q_d k_d| scale (the sum, the scale, the
              subtraction of the frame, whose own size adds e |s|), so p by the same
              amount relative (and 4 e for the exponential); p is rounded to the operand
              type (u), summed with the others (n e), and the result stored (u)
"""

import math

import torch

E32 = 2.0 ** -24


def unit(dt):
    return torch.finfo(dt).eps / 2


def seen(nq, nk, lq, lk, causal, window):
    i = torch.arange(nq)[:, None]
    j = torch.arange(nk)[None]
    p = i + lk - lq
    ok = (i < lq) & (j < lk)
    if causal:
        ok = ok & (j <= p)
    if window:
        ok = ok & (j > p - window)
    return ok


def attention(q, k, v, dout=None, causal=True, window=0, scale=None, lens_q=None, lens_k=None):
    """Values and bounds {name: (value, bound)} of out, lse and, with dout, dq, dk, dv."""
    u = unit(q.dtype)
    q, k, v = (x.detach().cpu() for x in (q, k, v))
    B, H, nq, D = q.shape
    Hkv, nk = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    f = torch.float64
    z = lambda *s: torch.zeros(*s, dtype=f)  # noqa: E731
    out, bo, lse, bl = z(B, H, nq, D), z(B, H, nq, D), torch.full((B, H, nq), -math.inf, dtype=f), z(B, H, nq)
    dq, bq = z(B, H, nq, D), z(B, H, nq, D)
    dk, bk, dv, bv = (z(B, Hkv, nk, D) for _ in range(4))
    for b in range(B):
        lq = nq if lens_q is None else min(max(int(lens_q[b]), 0), nq)
        lk = nk if lens_k is None else min(max(int(lens_k[b]), 0), nk)
        ok = seen(nq, nk, lq, lk, causal, window)
        for h in range(H):
            g = h // (H // Hkv)
            Q = torch.where(torch.arange(nq)[:, None] < lq, q[b, h].double(), 0.0)
            K = torch.where(torch.arange(nk)[:, None] < lk, k[b, g].double(), 0.0)
            V = torch.where(torch.arange(nk)[:, None] < lk, v[b, g].double(), 0.0)
            s = torch.where(ok, Q @ K.t() * scale, -math.inf)
            top = torch.where(ok.any(1), s.amax(1), 0.0)
            w = torch.exp(s - top[:, None])
            tot = w.sum(1)
            some = tot > 0
            p = w / torch.where(some, tot, 1.0)[:, None]
            ds_ = (D + 4) * E32 * (Q.abs() @ K.abs().t() * scale) + 4 * E32 * (1 + torch.where(ok, s, 0.0).abs())
            n = ok.sum(1)
            rel = ds_ + n[:, None] * E32                         # relative error of an unrounded p
            o = p @ V
            out[b, h] = o
            bo[b, h] = 1.01 * (u * o.abs() + (p * (u + 2 * rel)) @ V.abs()) + 1e-30
            lse[b, h] = torch.where(some, top + torch.log(torch.where(some, tot, 1.0)), -math.inf)
            bl[b, h] = 2 * rel.amax(1) + 8 * E32 * (1 + torch.where(some, lse[b, h], 0.0).abs())
            if dout is None:
                continue
            dO = torch.where(torch.arange(nq)[:, None] < lq, dout[b, h].detach().cpu().double(), 0.0)
            dp = dO @ V.t()
            delta = (dO * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            # delta from the stored out; dp, delta summed in float32
            bdel = (dO.abs() * bo[b, h]).sum(1, keepdim=True) + D * E32 * (dO.abs() * o.abs()).sum(1, keepdim=True)
            bdp = D * E32 * (dO.abs() @ V.abs().t())
            rp = rel + bl[b, h][:, None]
            bds = p * (bdel + bdp) + ds.abs() * (u + 2 * rp) + 1e-30
            dq[b, h] = scale * (ds @ K)
            bq[b, h] = 1.01 * (u * dq[b, h].abs() + scale * ((bds + ds.abs() * n[:, None] * E32) @ K.abs())) + 1e-30
            m = ok.sum(0).double() * (H // Hkv)
            dk[b, g] += scale * (ds.t() @ Q)
            bk[b, g] += 1.01 * scale * ((bds + ds.abs() * m[None] * E32).t() @ Q.abs())
            dv[b, g] += p.t() @ dO
            bv[b, g] += 1.01 * ((p * (u + 2 * rp + m[None] * E32)).t() @ dO.abs())
    bk += 1.01 * u * dk.abs() + 1e-30
    bv += 1.01 * u * dv.abs() + 1e-30
    got = {"out": (out, bo), "lse": (lse, bl)}
    return got if dout is None else {**got, "dq": (dq, bq), "dk": (dk, bk), "dv": (dv, bv)}


def recurrence(q, k, v, g, dout=None, s0=None, ds1=None, lens=None, scale=None):
    """Values and bounds of out, s1 and, with dout, dq, dk, dv, dg, ds0 (row by row)."""
    u = unit(q.dtype)
    us = u * u if q.dtype == torch.bfloat16 else u
    q, k, v, g = (x.detach().cpu().double().clone() for x in (q, k, v, g))
    B, H, n, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    ln = [n if lens is None else min(max(int(lens[b]), 0), n) for b in range(B)]
    do = None if dout is None else dout.detach().cpu().double().clone()
    for b in range(B):
        for x in (q, k, v, g) + (() if do is None else (do,)):
            x[b, :, ln[b]:] = 0
    slop = (4 * n + 200) * E32
    a = torch.exp(g)
    zero = torch.zeros(B, H, D, D, dtype=torch.float64)
    S = zero.clone() if s0 is None else s0.detach().cpu().double()
    A = S.abs()
    o, oa, dq, qa = (torch.zeros(B, H, n, D, dtype=torch.float64) for _ in range(4))
    before = []                                                # diag(a_t) |S|_{t-1} and diag(a_t) S_{t-1}
    for t in range(n):
        before.append((S * a[:, :, t, :, None], A * a[:, :, t, :, None]))
        S = before[t][0] + k[:, :, t, :, None] * v[:, :, t, None]
        A = before[t][1] + (k[:, :, t, :, None] * v[:, :, t, None]).abs()
        o[:, :, t] = scale * (q[:, :, t, :, None] * S).sum(2)
        oa[:, :, t] = abs(scale) * (q[:, :, t, :, None].abs() * A).sum(2)
        if do is not None:
            dq[:, :, t] = scale * (S * do[:, :, t, None]).sum(3)
            qa[:, :, t] = abs(scale) * (A * do[:, :, t, None].abs()).sum(3)
    for b in range(B):
        dq[b, :, ln[b]:] = 0
    tiny = 1e-30
    got = {"out": (o, 1.01 * (u * o.abs() + (3 * u + slop) * oa) + tiny), "s1": (S, 1.01 * (us + slop) * A + tiny)}
    if do is None:
        return got
    R = zero.clone() if ds1 is None else ds1.detach().cpu().double()
    Ra = R.abs()
    dk, ka, dv, va, dg, ga, ch = (torch.zeros(B, H, n, D, dtype=torch.float64) for _ in range(7))
    tail = torch.zeros(B, H, D, dtype=torch.float64)
    for t in range(n - 1, -1, -1):
        if t % 32 == 31 or t == n - 1:
            tail = (Ra * A if t == n - 1 else Ra * (before[t + 1][1] / a[:, :, t + 1, :, None].clamp_min(1e-300))).sum(3)
        R = R + scale * q[:, :, t, :, None] * do[:, :, t, None]
        Ra = Ra + abs(scale) * (q[:, :, t, :, None] * do[:, :, t, None]).abs()
        dk[:, :, t], ka[:, :, t] = (R * v[:, :, t, None]).sum(3), (Ra * v[:, :, t, None].abs()).sum(3)
        dv[:, :, t], va[:, :, t] = (R * k[:, :, t, :, None]).sum(2), (Ra * k[:, :, t, :, None].abs()).sum(2)
        dg[:, :, t], ga[:, :, t] = (R * before[t][0]).sum(3), (Ra * before[t][1]).sum(3)
        tail = tail + q[:, :, t].abs() * qa[:, :, t] + k[:, :, t].abs() * ka[:, :, t]
        ch[:, :, t] = tail
        R, Ra = R * a[:, :, t, :, None], Ra * a[:, :, t, :, None]
    for b in range(B):
        for x in (dk, dv, dg):
            x[b, :, ln[b]:] = 0
    return {**got, "dq": (dq, 1.01 * (u * dq.abs() + (3 * u + slop) * qa) + tiny),
            "dk": (dk, 1.01 * (u * dk.abs() + (3 * u + slop) * ka) + tiny),
            "dv": (dv, 1.01 * (u * dv.abs() + (3 * u + slop) * va) + tiny),
            # pairs that do not span a row cancel there to the float32 sums' error
            "dg": (dg, 1.01 * (u * dg.abs() + (5 * u + slop) * ga + slop * ch) + tiny),
            "ds0": (R, 1.01 * (us + slop) * Ra + tiny)}


def within(got, ref, name):
    """Asserts |got - value| <= bound elementwise (infinities equal)."""
    val, bound = ref
    x = got.detach().cpu().double()
    assert x.shape == val.shape, (name, x.shape, val.shape)
    inf = torch.isinf(val)
    assert torch.equal(x[inf], val[inf]), name
    d = (x - val).abs()[~inf]
    b = bound[~inf]
    assert bool(torch.isfinite(x[~inf]).all()), f"{name}: not finite"
    if d.numel():
        worst = (d / b).max().item()
        assert worst <= 1.0, f"{name}: {worst:.3g} times the bound"
