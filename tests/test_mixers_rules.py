"""Which kernel, how many pieces: the rules of the mixers' host side, as far as the
workspace's size shows them (no GPU needed)."""

import pytest

from paper_2608_09307_amd import linsimp as L


def pieces(d):
    """Pieces that the keys of a forward or a step are split into: each writes a row
    of D values, a maximum and a sum for every query (256-byte steps, two arrays)."""
    rows = d.B * d.H * d.nq
    size = L.attn_workspace_size(d, False)
    al = lambda x: -(-x // 256) * 256  # noqa: E731
    n = [n for n in range(2, 65) if al(n * rows * d.D * 4) + al(n * rows * 8) == size]
    return n[0] if n else 1


@pytest.mark.parametrize("B,H,Hkv,cap,D", [(8, 128, 1, 32768, 128), (16, 128, 1, 8192, 128), (1, 128, 1, 65536, 128),
                                          (4, 64, 1, 65536, 128), (4, 64, 8, 65536, 128), (1, 40, 1, 65536, 32)])
def test_a_step_of_few_heads_over_long_rings_fills_the_chip(B, H, Hkv, cap, D):
    """A workgroup of the step takes 32 heads of one key head: the pieces of the ring
    have to make up for the few of them, however many heads share a key head."""
    n = pieces(L.AttnDims(B, H, Hkv, 1, cap, 0, D, L.BF16, 1, 0.1))
    groups = B * Hkv * -(-(H // Hkv) // 32)
    assert groups * n >= 128, (groups, n)


def test_a_lone_workgroup_in_the_last_round_is_one_past_what_a_cu_holds():
    """D = 32: a CU holds five workgroups (float32: four), not three: 64 heads of 1000
    queries against 9000 keys take two pieces (136 us in two, 139 in three)."""
    for dt in (L.BF16, L.F32):
        assert pieces(L.AttnDims(4, 16, 4, 1000, 9000, 0, 32, dt, 1, 0.1)) == 2


def segments(d):
    """Segments of a forward of the recurrence: a word, and where there is more than one
    a state and a decay of each (256-byte steps)."""
    al = lambda x: -(-x // 256) * 256  # noqa: E731
    size, bh = L.glr_workspace_size(d, False), d.B * d.H
    n = [n for n in range(2, 257) if al(bh * n * 4) + al(bh * n * d.D * d.D * 4) + al(bh * n * d.D * 4) == size]
    return n[0] if n else 1


@pytest.mark.parametrize("D,dt,fits", [(32, L.BF16, 7), (64, L.BF16, 4), (128, L.BF16, 2), (64, L.F32, 3)])
@pytest.mark.parametrize("B,H,n", [(2, 16, 16384), (1, 8, 16384)])
def test_segments_fill_one_round_of_what_a_cu_holds(B, H, n, D, dt, fits):
    """Long sequences of a few heads: the shortest segments, in whole chunks of 32 rows,
    that run at once."""
    g, chunks = segments(L.GlrDims(B, H, n, D, dt, 0.1)), n // 32
    per = -(-chunks // g)
    assert B * H * g <= 256 * fits < B * H * -(-chunks // (per - 1)), (g, per)
