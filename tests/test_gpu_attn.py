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
