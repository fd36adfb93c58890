"""Attention with many query rows on one key head, so that a key head has several
sets of 32 columns, split over a long axis as well (definitions: mixer_ref)."""

import pytest
import torch

import mixer_ref as R
from test_gpu_attn import BF, DEV, F32, draw, step_ref
from paper_2608_09307_amd import linsimp as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hkv,cap,D,dt,pos", [
    (40, 1, 6000, 32, BF, [5999, 20000]), (70, 2, 5000, 64, BF, [4999, -1, 130]), (64, 1, 9000, 128, BF, [8999]),
    (66, 2, 4000, 32, F32, [3999, 17]), (33, 1, 3000, 64, F32, [1 << 40]),
])
def test_split_step_with_more_than_32_heads_on_a_key_head(H, Hkv, cap, D, dt, pos):
    print(f"[attn] split step {H, Hkv, cap, D, dt, pos}", flush=True)
    B = len(pos)
    q, kc, vc, _ = draw(B, H, Hkv, 1, cap, D, dt, seed=H)
    _, k, v, _ = draw(B, H, Hkv, 1, 1, D, dt, seed=H + 1)
    q, k, v = q[:, :, 0].contiguous(), k[:, :, 0].contiguous(), v[:, :, 0].contiguous()
    for b, p in enumerate(pos):                               # slots no token has reached
        if 0 <= p < cap:
            kc[b, :, p:], vc[b, :, p:] = float("nan"), float("inf")
    d = L.attn_dims(q[:, :, None], kc)
    assert L.attn_workspace_size(d, False) > 2 * B * H * D * 4, "not split"
    rk, rv, ref = step_ref(kc, vc, pos, q, k, v)
    out = L.attn_step(kc, vc, torch.tensor(pos, dtype=torch.int64, device=DEV), q, k, v)
    torch.cuda.synchronize()
    bits = lambda x: x.view(torch.int16 if dt == BF else torch.int32)  # noqa: E731  (unused slots hold NaN)
    assert torch.equal(bits(kc), bits(rk)) and torch.equal(bits(vc), bits(rv))
    R.within(out, ref, "out")


def kernels(q, k, v):
    """Names of the kernels of a forward, by the library's own timing."""
    L.attn_fwd(q, k, v)
    torch.cuda.synchronize()
    L.timing_enable(True)
    try:
        L.timing_read()                                       # (whatever an earlier user left)
        L.attn_fwd(q, k, v)
        torch.cuda.synchronize()
        return set(L.timing_read())
    finally:
        L.timing_enable(False)


@pytest.mark.parametrize("H,Hkv", [(1, 1), (8, 2), (16, 1)])
def test_the_few_row_kernel_takes_up_to_32_queries_of_a_head(H, Hkv):
    """However many heads share a key head: it reads the keys once per 32 columns, the
    other kernel once per head."""
    for nq, name in ((1, "attn_few"), (5, "attn_few"), (32, "attn_few"), (33, "attn_fwd")):
        q, k, v, _ = draw(1, H, Hkv, nq, 600, 64, BF)
        got = kernels(q, k, v)
        assert name in got and len(got - {"attn_join"}) == 1, (nq, got)


@pytest.mark.parametrize("dt,D", [(BF, 128), (BF, 64), (BF, 32), (F32, 64), (F32, 32)])
@pytest.mark.parametrize("H,Hkv,nq", [(8, 1, 20), (12, 2, 32), (3, 1, 31), (16, 2, 9)])
@pytest.mark.parametrize("window", [0, 33, 300])
def test_continuations_in_several_column_groups(H, Hkv, nq, D, dt, window):
    """More than 32 query rows on a key head, heads that straddle two groups of
    columns, with lengths; NaN and infinities behind the lengths."""
    print(f"[attn] columns {H} {Hkv} {nq} {D} {dt} {window}", flush=True)
    lq, lk = [nq, nq - 4, 1, 0], [1500, 333, 2, 40]
    x = draw(4, H, Hkv, nq, 1500, D, dt, seed=window + nq)
    ref = R.attention(*x, window=window, lens_q=lq, lens_k=lk)
    for b in range(4):
        for y, n in zip(x, (lq[b], lk[b], lk[b], lq[b])):
            y[b, :, n:] = float("nan")
            y[b, :, n + 1:] = float("inf")
    how = dict(window=window, lens_q=torch.tensor(lq, dtype=torch.int32, device=DEV),
               lens_k=torch.tensor(lk, dtype=torch.int32, device=DEV))
    out, lse = L.attn_fwd(*x[:3], **how)
    got = dict(zip(("dq", "dk", "dv"), L.attn_bwd(*x[:3], out, lse, x[3], **how)), out=out, lse=lse)
    torch.cuda.synchronize()
    for name in got:
        R.within(got[name], ref[name], name)


@pytest.mark.parametrize("H,Hkv,nq,nk,D,causal", [(8, 1, 32, 6000, 128, True), (40, 1, 3, 5000, 32, True), (6, 1, 30, 4000, 64, False)])
def test_long_continuations_in_pieces(H, Hkv, nq, nk, D, causal):
    print(f"[attn] column pieces {H} {Hkv} {nq} {nk} {D}", flush=True)
    q, k, v, _ = draw(1, H, Hkv, nq, nk, D, BF, seed=nk)
    assert L.attn_workspace_size(L.attn_dims(q, k, causal), False) > 2 * H * nq * D * 4, "not split"
    out, lse = L.attn_fwd(q, k, v, causal=causal)
    ref = R.attention(q, k, v, causal=causal)
    torch.cuda.synchronize()
    R.within(out, ref["out"], "out")
    R.within(lse, ref["lse"], "lse")
