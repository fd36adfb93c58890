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
