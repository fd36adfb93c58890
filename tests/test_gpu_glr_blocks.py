"""The bf16 recurrence on the GPU, block by block of 32 rows: the root mean square of
the errors against what independent roundings leave (mixer_rms), which a missing or
wrong term exceeds (test_mixer_rms)."""

import pytest
import torch

import mixer_ref as R
import mixer_rms as M
from test_gpu_glr import BF, CASES, DEV, draw, train

pytestmark = pytest.mark.gpu

LONG = [
    (1, 1, 3000, 64, BF, "mixed", True, None),
    (1, 1, 1500, 128, BF, "reset", True, None),
    (2, 2, 1200, 128, BF, "mixed", True, [1200, 517]),
    (1, 2, 1000, 128, BF, "slow", False, None),
    (1, 4, 900, 32, BF, "clear", True, None),
    (2, 3, 700, 64, BF, "none", True, [700, 290]),
]


@pytest.mark.parametrize("c", [c for c in CASES if c[4] == BF] + LONG,
                         ids=lambda c: "-".join(map(str, c[:4])) + f"-{c[5]}-{c[6]}")
def test_blocks(c):
    B, H, n, D, dt, kind, state, lens = c
    print(f"[glr] blocks {c}", flush=True)
    x = draw(B, H, n, D, dt, kind, state, seed=n + D + 1)
    got = train(x, None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV))
    ref = R.recurrence(x["q"], x["k"], x["v"], x["g"], x["dout"], x["s0"], x["ds1"], lens)
    bound = M.block_bounds(x, lens)
    worst = {name: (M.block_errors(got[name], ref[name][0]) / bound[name]).max().item() for name in bound}
    print({name: round(w, 3) for name, w in worst.items()}, flush=True)
    for name in bound:
        M.within_blocks(got[name], ref[name][0], bound[name], name)
