"""The block bounds of the recurrence's gradients against planted mistakes, on the
CPU: a missing term of dg has to show, and what rounding does must not."""

import pytest
import torch

import mixer_ref as R
import mixer_rms as M
from test_gpu_glr import BF, gates


def draw(B, H, n, D, kind, state, seed):
    gen = torch.Generator().manual_seed(seed)
    f = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x = {nm: f(B, H, n, D) for nm in ("q", "k", "v", "dout")}
    x["k"] *= D ** -0.5
    x["g"] = gates(kind, (B, H, n, D), gen)
    x = {nm: y.to(BF) for nm, y in x.items()}
    for nm in ("s0", "ds1"):
        x[nm] = f(B, H, D, D) if state else None
    return x


@pytest.mark.parametrize("n,D,kind", [(333, 64, "none"), (300, 128, "mixed"), (100, 64, "mixed"), (700, 32, "slow")])
def test_every_term_of_dg_counts(n, D, kind):
    x = draw(1, 1, n, D, kind, True, n)
    ref = R.recurrence(*(x[nm] for nm in "qkvg"), x["dout"], x["s0"], x["ds1"])["dg"]
    bound = M.block_bounds(x)["dg"]
    parts = M.dg_parts(x)
    whole = sum(parts.values())
    assert (whole - ref[0]).abs().max() <= 1e-10 * ref[0].abs().max()
    # a right result, rounded once at its store, is inside
    assert M.within_blocks(whole.to(BF), ref[0], bound, "dg") < 1
    for src, part in parts.items():
        if kind == "slow" and src == ("s0", "ds1"):            # (700 rows decay it by e^-35: there is no such term)
            continue
        off = M.block_errors(whole - part, ref[0]) / bound
        assert off.max() > 3, (src, off.max())
    # the elementwise bound lets a dg of zeros through at most elements of a long case
    assert (M.block_errors(torch.zeros_like(whole), ref[0]) / bound).min() > 3


@pytest.mark.parametrize("name", ["out", "dq", "dk", "dv"])
def test_a_missing_chunk_counts(name):
    """The other results without what the first chunk's rows of k, v (q, dout) add."""
    x = draw(1, 2, 300, 64, "mixed", True, 7)
    how = lambda y: R.recurrence(*(y[nm] for nm in "qkvg"), y["dout"], y["s0"], y["ds1"])[name][0]  # noqa: E731
    bound = M.block_bounds(x)[name]
    y = {nm: t.clone() if t is not None else None for nm, t in x.items()}
    cut = slice(64, 96) if name in ("out", "dq") else slice(200, 232)
    for nm in ("k", "v") if name in ("out", "dq") else ("q", "dout"):
        y[nm][:, :, cut] = 0
    off = M.block_errors(how(y), how(x)) / bound
    rest = [c for c in range(off.shape[2]) if not (cut.start // 32 <= c <= cut.stop // 32)]
    assert off[:, :, rest].max() > 3, off
