"""Softmax attention and the gated linear recurrence: sizes and refusals of the C
ABI and of the binding, before anything reaches a GPU."""

import ctypes
import math

import pytest
import torch

from paper_2608_09307_amd import linsimp as L

VP = ctypes.c_void_p
INF = math.inf


def attn(B=2, H=4, Hkv=2, nq=100, nk=100, window=0, D=64, dtype=L.BF16, causal=1, scale=0.125):
    return L.AttnDims(B, H, Hkv, nq, nk, window, D, dtype, causal, scale)


def glr(B=2, H=4, n=100, D=64, dtype=L.BF16, scale=0.125):
    return L.GlrDims(B, H, n, D, dtype, scale)


def message():
    return L.lib().linsimp_last_error().decode()


def ptrs(n, bad=None, value=0):
    p = [4096 * (i + 1) for i in range(n)]
    if bad is not None:
        p[bad] = value
    return [VP(x) for x in p]


def call(name, d, p, ws=1 << 20, size=1 << 40):
    return getattr(L.lib(), name)(ctypes.byref(d), *p, VP(ws), size, VP(0))


@pytest.mark.parametrize("change,status", [
    (dict(B=0), -1), (dict(H=0), -1), (dict(nq=0), -1), (dict(nk=-1), -1), (dict(H=3), -1), (dict(Hkv=8), -1),
    (dict(dtype=2), -1), (dict(causal=2), -1), (dict(window=-1), -1), (dict(window=4, causal=0), -1),
    (dict(scale=0.0), -1), (dict(scale=-1.0), -1), (dict(scale=INF), -1), (dict(scale=math.nan), -1),
    (dict(D=48), -2), (dict(D=128, dtype=L.F32), -2), (dict(D=256), -2),
    (dict(nk=(1 << 30) + 1), -2), (dict(B=1 << 20, H=2, Hkv=1), -2), (dict(B=1 << 16, nq=1 << 14), -2),
    (dict(B=1 << 62, H=1 << 62, Hkv=1), -2),
])
def test_attention_refuses_dims(change, status):
    d = attn(**change)
    assert L.attn_workspace_size(d, False) == 0 and message()
    assert call("linsimp_attn_fwd", d, ptrs(7)) == status and message()
    assert call("linsimp_attn_bwd", d, ptrs(11)) == status
    d.nq = 1 if "nq" not in change else d.nq
    assert call("linsimp_attn_step", d, ptrs(7)) < 0


def test_attention_refuses_pointers_and_workspaces():
    d = attn()
    for i in (0, 1, 2, 5):                                    # lens and lse may be NULL
        assert call("linsimp_attn_fwd", d, ptrs(7, i, 0)) == -1 and "NULL" in message()
        assert call("linsimp_attn_fwd", d, ptrs(7, i, 4104)) == -1 and "aligned" in message()
    assert call("linsimp_attn_fwd", d, ptrs(7, 3, 4098)) == -1 and "lens_q" in message()
    for i in (0, 1, 2, 5, 6, 7, 8, 9, 10):
        assert call("linsimp_attn_bwd", d, ptrs(11, i, 0)) == -1
    for i in range(7):
        assert call("linsimp_attn_step", attn(nq=1), ptrs(7, i, 0)) == -1
    assert call("linsimp_attn_step", attn(nq=2), ptrs(7)) == -1 and "nq" in message()
    assert call("linsimp_attn_step", attn(nq=1, window=8), ptrs(7)) == -1
    for name, n in (("linsimp_attn_fwd", 7), ("linsimp_attn_bwd", 11)):
        assert call(name, d, ptrs(n), ws=0) == -3
        assert call(name, d, ptrs(n), ws=4096 + 16) == -3
        assert call(name, d, ptrs(n), size=16) == -3 and "too small" in message()
    assert L.lib().linsimp_attn_fwd(None, *ptrs(7), VP(4096), 1 << 20, VP(0)) == -1


def test_attention_workspace_sizes():
    d = attn(B=1, H=16, Hkv=4, nq=1, nk=65536, D=128)
    one = L.attn_workspace_size(d, False)
    assert one > 0 and L.attn_workspace_size(d, True) >= one
    # the backward's limit on keys does not bind the forward
    big = attn(B=64, H=8, Hkv=8, nq=1, nk=1 << 22, D=32)
    assert L.attn_workspace_size(big, False) > 0
    assert L.attn_workspace_size(big, True) == 0 and "2^30" in message()
    # a window as wide as the keys is none
    assert L.attn_workspace_size(attn(window=100), True) == L.attn_workspace_size(attn(), True)


@pytest.mark.parametrize("change,status", [
    (dict(B=0), -1), (dict(H=-1), -1), (dict(n=0), -1), (dict(dtype=7), -1), (dict(scale=INF), -1),
    (dict(scale=math.nan), -1), (dict(D=16), -2), (dict(D=128, dtype=L.F32), -2),
    (dict(B=256, H=256), -2), (dict(n=(1 << 30) + 1), -2), (dict(B=1, H=3, n=1 << 30), -2),
    (dict(B=1 << 62, H=1 << 62), -2),
])
def test_recurrence_refuses_dims(change, status):
    d = glr(**change)
    assert L.glr_workspace_size(d, True) == 0 and message()
    assert call("linsimp_glr_fwd", d, ptrs(8)) == status and message()
    assert call("linsimp_glr_bwd", d, ptrs(13)) == status


def test_recurrence_refuses_pointers_and_workspaces():
    d = glr()
    for i in (0, 1, 2, 3, 6):
        assert call("linsimp_glr_fwd", d, ptrs(8, i, 0)) == -1 and "NULL" in message()
    for i in (4, 7):
        assert call("linsimp_glr_fwd", d, ptrs(8, i, 4100)) == -1 and "aligned" in message()
    for i in (0, 1, 2, 3, 6, 8, 9, 10, 11):
        assert call("linsimp_glr_bwd", d, ptrs(13, i, 0)) == -1
    for name, n in (("linsimp_glr_fwd", 8), ("linsimp_glr_bwd", 13)):
        assert call(name, d, ptrs(n), ws=0) == -3
        assert call(name, d, ptrs(n), size=16) == -3
    one = glr(n=1)
    assert L.lib().linsimp_glr_step(ctypes.byref(d), *ptrs(6), VP(0)) == -1 and "n must be 1" in message()
    for i in range(6):
        assert L.lib().linsimp_glr_step(ctypes.byref(one), *ptrs(6, i, 0), VP(0)) == -1
    # the step's grid holds more states than the others'
    assert L.lib().linsimp_glr_step(ctypes.byref(glr(B=1 << 20, H=16, n=1)), *ptrs(6), VP(0)) == -2
    assert L.lib().linsimp_glr_step(ctypes.byref(glr(B=1 << 10, H=1 << 10, n=1)), *ptrs(6, 0, 0), VP(0)) == -1


def test_binding_refuses_tensors():
    q = torch.zeros(1, 2, 8, 32)
    k = torch.zeros(1, 2, 8, 32)
    with pytest.raises(ValueError, match="GPU"):
        L.attn_fwd(q, k, k)
    with pytest.raises(ValueError, match="GPU"):
        L.glr_fwd(q, k, k, k)
    with pytest.raises(TypeError):
        L.attn_fwd(q.half(), k.half(), k.half())
    with pytest.raises(ValueError, match="shape"):
        L.attn_fwd(q, k, k[:, :, :4])
    with pytest.raises(TypeError, match="dtype"):
        L.attn_fwd(q, k.bfloat16(), k)
    with pytest.raises(TypeError, match="lens_q"):
        L.attn_fwd(q, k, k, lens_q=torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError, match="lens"):
        L.glr_fwd(q, k, k, k, lens=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        L.attn_fwd(q[0], k, k)
    with pytest.raises(ValueError):
        L.glr_step(torch.zeros(1, 2, 32, 32), q, k, k, k)
    with pytest.raises(ValueError, match="shape"):
        L.glr_step(torch.zeros(1, 2, 32, 16), q[:, :, 0], k[:, :, 0], k[:, :, 0], k[:, :, 0])
    with pytest.raises(TypeError, match="pos"):
        L.attn_step(k, k.clone(), torch.zeros(1, dtype=torch.int32), q[:, :, 0], k[:, :, 0], k[:, :, 0])
    # refused dims come back as the library's error, with its message
    with pytest.raises(L.LinSimpError, match="Hkv"):
        L._mixer_workspace(None, L.attn_workspace_size(attn(H=3), False), torch.device("cpu"))
