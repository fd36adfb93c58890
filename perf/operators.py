"""Timing cases of the two mixers that stand beside the LinSimp core in a hybrid
stack: softmax attention (forward, backward from recomputed probabilities, and
the single-token step on a ring cache) and the gated linear recurrence (forward
with its state, backward, and the single-token step).

With ``own`` false, ``run`` computes them in elementary torch operations in 32
bits; with ``own`` true it makes the calls a user's program makes of
``paper_2608_09307_amd.linsimp``.

    attention    o_i = sum_j p_ij v_j,  p_i = softmax_j(scale q_i . k_j) over the visible j
    recurrence   S_t = diag(exp(g_t)) S_{t-1} + k_t v_t^T,  o_t = scale S_t^T q_t

A case is a dict of plain values:
  op      "attn_fwd"   out, lse                (scoring, prefill of a prompt)
          "attn_train" out, lse, dq, dk, dv
          "attn_step"  one token for every sequence, on a ring of cap slots
          "glr_fwd"    out and the state after the last token
          "glr_train"  out, dq, dk, dv, dg, and with state the final state and ds0
          "glr_step"   one token for every sequence
  B (sequences), H (heads), D (head width), dtype "bf16" or "f32"
  attention: Hkv (heads of k and v), nq, nk, causal, window (0: none), ragged; cap
  recurrence: n, ragged, state (starts from a state), gate ("slow", "mixed", "reset")
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda"
CHUNK = 32            # rows per block of the plain recurrence


def listed():
    return [
        # one interactive stream of a small model: a token at a time, latency
        dict(name="attn_step_1seq", op="attn_step", B=1, H=6, Hkv=6, D=64, cap=2048, dtype="bf16"),
        # batched serving after long prompts, four query heads per key head
        dict(name="attn_step_256seq", op="attn_step", B=256, H=16, Hkv=4, D=128, cap=8192, dtype="bf16"),
        # a few long sessions: few rows, a long axis
        dict(name="attn_step_4seq_64k", op="attn_step", B=4, H=16, Hkv=2, D=128, cap=65536, dtype="bf16"),
        # the next 1000 tokens of long prompts, against what is cached already
        dict(name="attn_prefill_chunk", op="attn_fwd", B=2, H=16, Hkv=4, nq=1000, nk=9000, D=128, causal=True,
             window=0, ragged=True, dtype="bf16"),
        # training step of the 2k-token layer
        dict(name="attn_train_2k", op="attn_train", B=8, H=6, Hkv=6, nq=2048, nk=2048, D=64, causal=True, window=0,
             ragged=False, dtype="bf16"),
        # training step of the 16k-token layer
        dict(name="attn_train_16k", op="attn_train", B=1, H=16, Hkv=16, nq=16384, nk=16384, D=128, causal=True,
             window=0, ragged=False, dtype="bf16"),
        # gradient checks and small models: float32, shared heads, odd sizes, a window, a padded batch
        dict(name="attn_train_f32_n777", op="attn_train", B=3, H=4, Hkv=2, nq=777, nk=777, D=32, causal=True,
             window=129, ragged=True, dtype="f32"),
        # batched serving: a token for every sequence
        dict(name="glr_step_256seq", op="glr_step", B=256, H=16, D=128, gate="mixed", dtype="bf16"),
        # a padded batch of prompts, to the state that decoding starts from
        dict(name="glr_prefill_8k", op="glr_fwd", B=4, H=16, n=8192, D=128, ragged=True, state=False, gate="mixed",
             dtype="bf16"),
        # training step of the 2k-token layer
        dict(name="glr_train_2k", op="glr_train", B=8, H=6, n=2048, D=64, ragged=False, state=False, gate="slow",
             dtype="bf16"),
        # training step of the 16k-token layer
        dict(name="glr_train_16k", op="glr_train", B=2, H=16, n=16384, D=128, ragged=False, state=False, gate="mixed",
             dtype="bf16"),
        # float32, odd length, a padded batch, gates that clear the state, a state carried in and out
        dict(name="glr_train_f32_n777", op="glr_train", B=3, H=4, n=777, D=32, ragged=True, state=True, gate="reset",
             dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attn_fwd", "attn_train", "attn_train", "attn_step", "attn_step",
                     "glr_fwd", "glr_train", "glr_train", "glr_step"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    D = rng.choice((32, 64) if dtype == "f32" else (32, 64, 128))
    H = rng.choice((1, 2, 4, 6, 8, 12, 16, 32))
    c = dict(op=op, B=_log_int(rng, 1, 64), H=H, D=D, dtype=dtype)
    if op == "glr_step":
        c["B"] = _log_int(rng, 1, 256)
        c["gate"] = rng.choice(("slow", "mixed", "reset"))
        return c
    if op.startswith("attn"):
        c["Hkv"] = rng.choice([h for h in (1, 2, 3, 4, 6, 8, 12, 16, 32) if H % h == 0])
    if op == "attn_step":
        c["B"] = _log_int(rng, 1, 256)
        c["cap"] = _log_int(rng, 16, 65536)
        while c["B"] * c["Hkv"] * c["cap"] * c["D"] > 1 << 30:
            c["B"] = max(1, c["B"] // 2)
            c["cap"] = max(16, c["cap"] * 3 // 4)
        return c
    # (one visible key has no gradient to compare: training starts at a few rows)
    n = _log_int(rng, 16 if op == "attn_train" else 2 if op == "glr_train" else 1, 16384)
    c["ragged"] = rng.random() < 0.4
    if op.startswith("glr"):
        c["n"] = n
        c["state"] = rng.random() < 0.3
        c["gate"] = rng.choice(("slow", "mixed", "mixed", "reset"))
        while c["B"] * H * n * D > 1 << 26 and c["B"] > 1:
            c["B"] -= 1
        while c["B"] * H * n * D > 1 << 26:
            n = c["n"] = n // 2 + 1
        return c
    c["nq"] = n
    c["nk"] = n if rng.random() < 0.7 else n + _log_int(rng, 1, 8192)
    c["causal"] = rng.random() < 0.85
    c["window"] = _log_int(rng, 8, 4096) if c["causal"] and rng.random() < 0.3 else 0
    most = 1 << 32 if dtype == "bf16" else 1 << 30
    while c["B"] * H * c["nq"] * c["nk"] > most and c["B"] > 1:
        c["B"] -= 1
    while c["B"] * H * c["nq"] * c["nk"] > most:
        c["nq"], c["nk"] = c["nq"] // 2 + 1, c["nk"] // 2 + 1
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _dt(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _spread(B, n):
    """Lengths of a padded batch: from n down to about n / 2."""
    return [max(1, n - (b * n) // (2 * B)) for b in range(B)]


def _lens(c):
    """(lens_q, lens_k) of an attention case, as lists."""
    B, nq, nk = c["B"], c["nq"], c["nk"]
    if not c["ragged"]:
        return [nq] * B, [nk] * B
    lq = _spread(B, nq)
    return lq, [nk - (nq - x) for x in lq]


def _positions(c):
    """Index of the new token of every sequence: from a quarter of the ring to past its end."""
    B, cap = c["B"], c["cap"]
    return [(cap // 4 + (b * cap) // B + 7 * b) if B > 1 else cap - 1 for b in range(B)]


def _gates(c, shape, gen):
    """Log decays: "slow" as a logsigmoid over 16, "mixed" with a time constant per
    channel between 1 and 4096 rows, "reset" the same with one row in 64 at -40."""
    x = torch.randn(shape, generator=gen, device=DEV)
    if c["gate"] == "slow":
        return torch.nn.functional.logsigmoid(x) / 16
    rate = torch.exp(-math.log(4096.0) * torch.rand(shape[-1], generator=gen, device=DEV))
    g = -rate * torch.exp(0.5 * x)
    if c["gate"] == "reset":
        g = torch.where(torch.rand(shape, generator=gen, device=DEV) < 1 / 64, torch.full_like(g, -40.0), g)
    return g


def prepare(case, seed):
    c, op, dt = case, case["op"], _dt(case)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEV, dtype=dt)

    def lens(v):
        return torch.tensor(v, dtype=torch.int32, device=DEV)

    B, H, D = c["B"], c["H"], c["D"]
    st = {"case": c, "scale": D ** -0.5}
    if op == "attn_step":
        Hkv, cap = c["Hkv"], c["cap"]
        st.update(q=normal(B, H, D), k=normal(B, Hkv, D), v=normal(B, Hkv, D), kc=normal(B, Hkv, cap, D),
                  vc=normal(B, Hkv, cap, D), pos=torch.tensor(_positions(c), dtype=torch.int64, device=DEV))
        return st
    if op == "glr_step":
        st.update(q=normal(B, H, D), k=normal(B, H, D) * D ** -0.5, v=normal(B, H, D),
                  g=_gates(c, (B, H, D), gen).to(dt),
                  state=torch.randn((B, H, D, D), generator=gen, device=DEV))
        return st
    if op.startswith("attn"):
        st.update(q=normal(B, H, c["nq"], D), k=normal(B, c["Hkv"], c["nk"], D), v=normal(B, c["Hkv"], c["nk"], D))
        if c["ragged"]:
            st["lens_q"], st["lens_k"] = (lens(x) for x in _lens(c))
        if op == "attn_train":
            st["dout"] = normal(B, H, c["nq"], D)
        return st
    n = c["n"]
    st.update(q=normal(B, H, n, D), k=normal(B, H, n, D) * D ** -0.5, v=normal(B, H, n, D),
              g=_gates(c, (B, H, n, D), gen).to(dt))
    if c["ragged"]:
        st["lens"] = lens(_spread(B, n))
    if c["state"]:
        st["s0"] = torch.randn((B, H, D, D), generator=gen, device=DEV)
    if op == "glr_train":
        st["dout"] = normal(B, H, n, D)
        if c["state"]:
            st["ds1"] = torch.randn((B, H, D, D), generator=gen, device=DEV)
    return st


# ---------------------------------------------------------------------------
# The framework's calls
# ---------------------------------------------------------------------------

def _run_own(st):
    from paper_2608_09307_amd import linsimp as L

    c, op, scale = st["case"], st["case"]["op"], st["scale"]
    if op == "glr_step":
        out = L.glr_step(st["state"], st["q"], st["k"], st["v"], st["g"], scale=scale)
        return {"out": out, "state": st["state"]}
    if "workspace" not in st:                         # the program keeps its workspace from its first call on
        if op == "attn_step":
            d = L.attn_dims(st["q"].unsqueeze(2), st["kc"], scale=scale)
        elif op.startswith("attn"):
            d = L.attn_dims(st["q"], st["k"], causal=c["causal"], window=c["window"], scale=scale)
        else:
            d = L.glr_dims(st["q"], scale=scale)
        size = L.glr_workspace_size if op.startswith("glr") else L.attn_workspace_size
        st["workspace"] = L.alloc_bytes(size(d, op.endswith("train")), st["q"].device)
    ws = st["workspace"]
    if op == "attn_step":
        out = L.attn_step(st["kc"], st["vc"], st["pos"], st["q"], st["k"], st["v"], scale=scale, workspace=ws)
        return {"out": out, "kc": st["kc"], "vc": st["vc"]}
    if op.startswith("attn"):
        how = dict(causal=c["causal"], window=c["window"], scale=scale, lens_q=st.get("lens_q"),
                   lens_k=st.get("lens_k"), workspace=ws)
        out, lse = L.attn_fwd(st["q"], st["k"], st["v"], **how)
        if op == "attn_fwd":
            return {"out": out, "lse": lse}
        dq, dk, dv = L.attn_bwd(st["q"], st["k"], st["v"], out, lse, st["dout"], **how)
        return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    x = (st["q"], st["k"], st["v"], st["g"])
    how = dict(scale=scale, s0=st.get("s0"), lens=st.get("lens"), workspace=ws)
    if op == "glr_fwd":
        out, s1 = L.glr_fwd(*x, **how)
        return {"out": out, "s1": s1}
    out, s1 = L.glr_fwd(*x, want_state=c["state"], **how)
    dq, dk, dv, dg, ds0 = L.glr_bwd(*x, st["dout"], ds1=st.get("ds1"), **how)
    got = {"out": out, "dq": dq, "dk": dk, "dv": dv, "dg": dg}
    return {**got, "s1": s1, "ds0": ds0} if c["state"] else got


# ---------------------------------------------------------------------------
# Plain forms (32 bits)
# ---------------------------------------------------------------------------

def _visible(c, st):
    """[B or 1, nq, nk]: whether query i sees key j."""
    nq, nk = c["nq"], c["nk"]
    i = torch.arange(nq, device=DEV)[:, None]
    j = torch.arange(nk, device=DEV)[None, :]
    lq = st["lens_q"][:, None, None] if c["ragged"] else torch.full((1, 1, 1), nq, device=DEV)
    lk = st["lens_k"][:, None, None] if c["ragged"] else torch.full((1, 1, 1), nk, device=DEV)
    ok = (i < lq) & (j < lk)
    if c["causal"]:
        p = i + (lk - lq)
        ok = ok & (j <= p)
        if c["window"]:
            ok = ok & (j > p - c["window"])
    return ok


def _plain_attn(st):
    c, dt = st["case"], _dt(st["case"])
    B, H, Hkv, nq, nk, D = c["B"], c["H"], c["Hkv"], c["nq"], c["nk"], c["D"]
    G = H // Hkv
    hidden = ~_visible(c, st)[:, None, None]
    q, k, v = st["q"].float().view(B, Hkv, G * nq, D), st["k"].float(), st["v"].float()
    s = (q * st["scale"]) @ k.transpose(2, 3)
    sg = s.view(B, Hkv, G, nq, nk)
    sg.masked_fill_(hidden, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    lse = (top + total.log()).view(B, H, nq)
    s.div_(torch.where(total == 0, torch.ones_like(total), total))
    out = s @ v
    got = {"out": out.view(B, H, nq, D).to(dt), "lse": lse}
    if c["op"] == "attn_fwd":
        return got
    do = st["dout"].float().view(B, Hkv, G * nq, D)
    got["dv"] = (s.transpose(2, 3) @ do).to(dt)
    delta = (do * out).sum(-1, keepdim=True)
    ds = do @ v.transpose(2, 3)
    ds.sub_(delta).mul_(s).mul_(st["scale"])
    got["dq"] = (ds @ k).view(B, H, nq, D).to(dt)
    got["dk"] = (ds.transpose(2, 3) @ q).to(dt)
    return got


def _plain_attn_step(st):
    c, dt = st["case"], _dt(st["case"])
    B, H, Hkv, cap, D = c["B"], c["H"], c["Hkv"], c["cap"], c["D"]
    pos, kc, vc = st["pos"], st["kc"], st["vc"]
    at = torch.arange(B, device=DEV)
    kc[at, :, pos % cap] = st["k"]
    vc[at, :, pos % cap] = st["v"]
    hidden = torch.arange(cap, device=DEV)[None] > pos[:, None]        # slots no token has reached
    q = st["q"].float().view(B, Hkv, H // Hkv, D) * st["scale"]
    s = q @ kc.float().transpose(2, 3)
    s.masked_fill_(hidden[:, None, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    out = (p @ vc.float()) / p.sum(-1, keepdim=True)
    return {"out": out.view(B, H, D).to(dt), "kc": kc, "vc": vc}


def _plain_glr(st, x, s0):
    """out, final state in 32 bits, from float32 leaves x = (q, k, v, g): blocks of
    CHUNK rows, each against the pairs inside it and the state before it."""
    c = st["case"]
    B, H, n, D = c["B"], c["H"], c["n"], c["D"]
    N = -(-n // CHUNK)
    if c["ragged"]:
        ok = (torch.arange(n, device=DEV)[None] < st["lens"][:, None])[:, None, :, None]
        x = [torch.where(ok, t, torch.zeros_like(t)) for t in x]
    q, k, v, g = (torch.nn.functional.pad(t, (0, 0, 0, N * CHUNK - n)).view(B, H, N, CHUNK, D) for t in x)
    G = g.double().cumsum(3)
    later = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=DEV).triu(1)[..., None]
    decay = (G[:, :, :, :, None] - G[:, :, :, None, :]).masked_fill(later, -math.inf).float().exp()
    p = (q[:, :, :, :, None] * (k[:, :, :, None, :] * decay)).sum(-1)
    # chunk contributions, then the state at every boundary
    total = G[:, :, :, -1]
    part = (k * (total[:, :, :, None] - G).float().exp()).transpose(3, 4) @ v       # [B, H, N, D, D]
    A = torch.nn.functional.pad(total.cumsum(2), (0, 0, 1, 0))                       # [B, H, N + 1, D]
    over = (A.transpose(2, 3)[..., :, None] - A[:, :, 1:].transpose(2, 3)[..., None, :])
    ahead = torch.ones(N + 1, N, dtype=torch.bool, device=DEV).triu(0)
    over = over.masked_fill(ahead, -math.inf).float().exp()                          # [B, H, D, N + 1, N]
    S = (over @ part.permute(0, 1, 3, 2, 4)).permute(0, 1, 3, 2, 4)                   # [B, H, N + 1, D, D]
    if s0 is not None:
        S = S + A.float().exp()[..., None] * s0[:, :, None]
    out = p @ v + (q * G.float().exp()) @ S[:, :, :-1]
    return out.reshape(B, H, N * CHUNK, D)[:, :, :n] * st["scale"], S[:, :, -1]


def _run_plain_glr(st):
    c, dt = st["case"], _dt(st["case"])
    names = ("q", "k", "v", "g")
    if c["op"] == "glr_fwd":
        out, s1 = _plain_glr(st, [st[x].float() for x in names], st.get("s0"))
        return {"out": out.to(dt), "s1": s1}
    leaves = [st[x].float().requires_grad_() for x in names]
    s0 = st["s0"].clone().requires_grad_() if c["state"] else None
    out, s1 = _plain_glr(st, leaves, s0)
    ends = ([out, s1], [st["dout"].float(), st["ds1"]]) if c["state"] else ([out], [st["dout"].float()])
    grads = torch.autograd.grad(ends[0], leaves + ([s0] if c["state"] else []), ends[1])
    got = {"out": out.detach().to(dt), "dq": grads[0].to(dt), "dk": grads[1].to(dt), "dv": grads[2].to(dt),
           "dg": grads[3].to(dt)}
    return {**got, "s1": s1.detach(), "ds0": grads[4]} if c["state"] else got


def _plain_glr_step(st):
    c, dt, S = st["case"], _dt(st["case"]), st["state"]
    S.mul_(st["g"].float().exp()[..., None]).add_(st["k"].float()[..., None] * st["v"].float()[..., None, :])
    out = (st["q"].float() * st["scale"])[:, :, None] @ S
    return {"out": out.squeeze(2).to(dt), "state": S}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "attn_step":
        return _plain_attn_step(state)
    if op == "glr_step":
        return _plain_glr_step(state)
    return _plain_attn(state) if op.startswith("attn") else _run_plain_glr(state)


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    """Each input read once, each output written once (the rows that exist, the slots
    that hold a token); the products of the visible pairs and of the state updates."""
    c, op = case, case["op"]
    e = 2 if c["dtype"] == "bf16" else 4
    B, H, D = c["B"], c["H"], c["D"]
    if op == "attn_step":
        seen = sum(min(p + 1, c["cap"]) for p in _positions(c))
        return {"bytes": e * D * (2 * B * H + 4 * B * c["Hkv"] + 2 * c["Hkv"] * seen), "flops": 4 * D * H * seen}
    if op == "glr_step":
        return {"bytes": B * H * (e * 5 * D + 2 * 4 * D * D), "flops": B * H * 5 * D * D}
    if op.startswith("attn"):
        pairs = rows = keys = 0
        for lq, lk in zip(*_lens(c)):
            p = np.arange(lq) + lk - lq
            hi = np.minimum(p, lk - 1) if c["causal"] else np.full(lq, lk - 1)
            lo = np.maximum(0, p - c["window"] + 1) if c["window"] else np.zeros(lq, np.int64)
            pairs += H * int(np.maximum(0, hi - lo + 1).sum())
            rows += H * lq
            keys += c["Hkv"] * lk
        if op == "attn_fwd":
            return {"bytes": e * D * (2 * rows + 2 * keys) + 4 * rows, "flops": 4 * D * pairs}
        return {"bytes": e * D * (4 * rows + 4 * keys) + 4 * rows, "flops": 14 * D * pairs}
    rows = H * (sum(_spread(B, c["n"])) if c["ragged"] else B * c["n"])
    states = B * H * D * D * 4
    if op == "glr_fwd":
        return {"bytes": e * D * 5 * rows + states * (2 if c["state"] else 1), "flops": rows * 5 * D * D}
    return {"bytes": e * D * 10 * rows + (4 * states if c["state"] else 0), "flops": rows * 16 * D * D}


# ---------------------------------------------------------------------------
# 64-bit values from the definitions
# ---------------------------------------------------------------------------

def _exact_attn(c, seed):
    st = prepare(c, seed)
    B, H, Hkv, nq, nk, D = c["B"], c["H"], c["Hkv"], c["nq"], c["nk"], c["D"]
    train = c["op"] == "attn_train"
    f64 = torch.float64
    out = torch.zeros(B, H, nq, D, dtype=f64, device=DEV)
    lse = torch.full((B, H, nq), -math.inf, dtype=f64, device=DEV)
    dq, dk, dv = torch.zeros_like(out), torch.zeros(B, Hkv, nk, D, dtype=f64, device=DEV), None
    dv = torch.zeros_like(dk)
    for b, (lq, lk) in enumerate(zip(*_lens(c))):
        rows = max(1, min(lq, (1 << 27) // max(1, lk)))
        j = torch.arange(lk, device=DEV)
        for h in range(H):
            kh = h // (H // Hkv)
            k, v = st["k"][b, kh, :lk].double(), st["v"][b, kh, :lk].double()
            for r0 in range(0, lq, rows):
                r1 = min(lq, r0 + rows)
                q = st["q"][b, h, r0:r1].double()
                at = (torch.arange(r0, r1, device=DEV) + lk - lq)[:, None]
                seen = torch.ones(r1 - r0, lk, dtype=torch.bool, device=DEV)
                if c["causal"]:
                    seen = j[None] <= at
                if c["window"]:
                    seen = seen & (at - j[None] < c["window"])
                s = torch.where(seen, q @ k.t().contiguous() * st["scale"], torch.tensor(-math.inf, dtype=f64, device=DEV))
                z = torch.logsumexp(s, 1)
                p = torch.where(seen, torch.exp(s - z[:, None]), torch.zeros((), dtype=f64, device=DEV))
                out[b, h, r0:r1] = p @ v
                lse[b, h, r0:r1] = z
                if train:
                    do = st["dout"][b, h, r0:r1].double()
                    dp = do @ v.t().contiguous()
                    ds = p * (dp - (p * dp).sum(1, keepdim=True)) * st["scale"]
                    dq[b, h, r0:r1] = ds @ k
                    dk[b, kh, :lk] += ds.t().contiguous() @ q
                    dv[b, kh, :lk] += p.t().contiguous() @ do
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv} if train else {"out": out, "lse": lse}


def _exact_attn_step(c, seed):
    st = prepare(c, seed)
    B, H, Hkv, cap = c["B"], c["H"], c["Hkv"], c["cap"]
    out = torch.empty(B, H, c["D"], dtype=torch.float64, device=DEV)
    for b, p in enumerate(_positions(c)):
        kc, vc = st["kc"][b], st["vc"][b]
        kc[:, p % cap], vc[:, p % cap] = st["k"][b], st["v"][b]
        m = min(p + 1, cap)
        q = st["q"][b].double().view(Hkv, H // Hkv, -1)
        w = torch.softmax(q @ kc[:, :m].double().transpose(1, 2) * st["scale"], -1)
        out[b] = (w @ vc[:, :m].double()).view(H, -1)
    return {"out": out, "kc": st["kc"], "vc": st["vc"]}


def _exact_glr(c, seed):
    """The recurrence itself, a row at a time: forward for S, out and dq; backward
    for R = d/dS, dk, dv; and g's gradient from d/dg_t = d/dg_{t+1} + q_t dq_t - k_t dk_t."""
    st = prepare(c, seed)
    B, H, n, D, scale = c["B"], c["H"], c["n"], c["D"], st["scale"]
    train = c["op"] == "glr_train"
    f64 = torch.float64
    x = {t: st[t].double() for t in ("q", "k", "v", "g") + (("dout",) if train else ())}
    if c["ragged"]:
        for b, m in enumerate(_spread(B, n)):
            for t in x.values():
                t[b, :, m:] = 0
    x = {t: y.permute(2, 0, 1, 3).contiguous() for t, y in x.items()}
    a = x["g"].exp()
    S = st["s0"].double() if c["state"] else torch.zeros(B, H, D, D, dtype=f64, device=DEV)
    out, dq = torch.empty(n, B, H, D, dtype=f64, device=DEV), torch.zeros(n, B, H, D, dtype=f64, device=DEV)
    for t in range(n):
        S = S * a[t][..., None] + x["k"][t][..., None] * x["v"][t][..., None, :]
        out[t] = (x["q"][t][..., None, :] @ S).squeeze(-2) * scale
        if train:
            dq[t] = (S @ x["dout"][t][..., None]).squeeze(-1) * scale
    back = lambda y: y.permute(1, 2, 0, 3)  # noqa: E731
    if not train:
        return {"out": back(out), "s1": S}
    R = st["ds1"].double() if c["state"] else torch.zeros(B, H, D, D, dtype=f64, device=DEV)
    dg_next = (R * S).sum(-1)
    dk, dv, dg = torch.empty_like(dq), torch.empty_like(dq), torch.empty_like(dq)
    for t in range(n - 1, -1, -1):
        R = R + x["q"][t][..., None] * x["dout"][t][..., None, :] * scale
        dk[t] = (R @ x["v"][t][..., None]).squeeze(-1)
        dv[t] = (x["k"][t][..., None, :] @ R).squeeze(-2)
        dg_next = dg_next + x["q"][t] * dq[t] - x["k"][t] * dk[t]
        dg[t] = dg_next
        R = R * a[t][..., None]
    got = {"out": back(out), "dq": back(dq), "dk": back(dk), "dv": back(dv), "dg": back(dg)}
    if c["ragged"]:
        for b, m in enumerate(_spread(B, n)):
            for t in ("dq", "dk", "dv", "dg"):
                got[t][b, :, m:] = 0
    return {**got, "s1": S, "ds0": R} if c["state"] else got


def _exact_glr_step(c, seed):
    st = prepare(c, seed)
    S = st["state"].double() * st["g"].double().exp()[..., None]
    S += st["k"].double()[..., None] * st["v"].double()[..., None, :]
    out = (S * st["q"].double()[..., None]).sum(-2) * st["scale"]
    return {"out": out, "state": S}


def exact(case, seed):
    op = case["op"]
    if op == "attn_step":
        return _exact_attn_step(case, seed)
    if op == "glr_step":
        return _exact_glr_step(case, seed)
    return _exact_attn(case, seed) if op.startswith("attn") else _exact_glr(case, seed)
