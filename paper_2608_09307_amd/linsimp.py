"""Thin ctypes binding of liblinsimp.so (the C ABI in include/linsimp.h,
include/linsimp_head.h and include/linsimp_bank.h).

Argument marshalling only: torch tensors are turned into device pointers and
the current HIP stream is passed through.  Every step of the computation runs
in the library's HIP kernels; there is no CPU or PyTorch fallback, and every
entry point raises if the library is not built or a tensor is not on the GPU.
"""

from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_lib", "liblinsimp.so")
_lib = None

F32, BF16 = 0, 1
EPS = 1e-30


class LinSimpError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"linsimp status {status}: {message}")
        self.status = status


class Dims(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("H", ctypes.c_int64), ("n", ctypes.c_int64),
                ("D", ctypes.c_int32), ("Dv", ctypes.c_int32), ("m", ctypes.c_int32),
                ("w", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


class AttnDims(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("H", ctypes.c_int64), ("Hkv", ctypes.c_int64),
                ("nq", ctypes.c_int64), ("nk", ctypes.c_int64), ("window", ctypes.c_int64),
                ("D", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class GlrDims(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int64), ("H", ctypes.c_int64), ("n", ctypes.c_int64),
                ("D", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class HeadOpts(ctypes.Structure):
    _fields_ = [("norm_eps", ctypes.c_float), ("rms_eps", ctypes.c_float), ("gate", ctypes.c_int32)]


GATE_HEAD, GATE_CHANNEL = 0, 1
NORM_EPS, RMS_EPS = 1e-12, 1e-6

BWD_REUSE_STATES = 1

EXPORTS = ("linsimp_workspace_size", "linsimp_fwd", "linsimp_fwd_static", "linsimp_bwd", "linsimp_bwd_ex",
           "linsimp_prefill",
           "linsimp_decode_step", "linsimp_decode_chunk",
           "linsimp_attn_workspace_size", "linsimp_attn_fwd", "linsimp_attn_bwd", "linsimp_attn_step",
           "linsimp_glr_workspace_size", "linsimp_glr_fwd", "linsimp_glr_bwd", "linsimp_glr_step",
           "linsimp_timing_enable",
           "linsimp_timing_read", "linsimp_last_error", "linsimp_version")
HEAD_EXPORTS = ("linsimp_head_saved_size", "linsimp_head_workspace_size", "linsimp_head_fwd",
                "linsimp_head_bwd", "linsimp_head_bwd_ex")
BANK_EXPORTS = ("linsimp_feature_bank",)


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Load liblinsimp.so (raises if it is not built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise RuntimeError(f"{_LIB_PATH} is not built; run paper_2608_09307_amd.build.build()")
    L = ctypes.CDLL(_LIB_PATH)
    vp, sz, i32, i64, f32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
    pd = ctypes.POINTER(Dims)
    L.linsimp_workspace_size.argtypes = [pd, ctypes.c_int]
    L.linsimp_workspace_size.restype = sz
    L.linsimp_fwd.argtypes = [pd] + [vp] * 8 + [vp, sz, vp]
    L.linsimp_fwd.restype = ctypes.c_int
    L.linsimp_fwd_static.argtypes = [pd] + [vp] * 8 + [vp]
    L.linsimp_fwd_static.restype = ctypes.c_int
    L.linsimp_bwd.argtypes = [pd] + [vp] * 14 + [vp, sz, vp]
    L.linsimp_bwd.restype = ctypes.c_int
    L.linsimp_bwd_ex.argtypes = [pd] + [vp] * 14 + [i32, vp, sz, vp]
    L.linsimp_bwd_ex.restype = ctypes.c_int
    L.linsimp_prefill.argtypes = [pd] + [vp] * 11 + [vp, sz, vp]
    L.linsimp_prefill.restype = ctypes.c_int
    L.linsimp_decode_step.argtypes = [i64, i32, i32, i32, i32, i32, i32, f32] + [vp] * 13 + [vp]
    L.linsimp_decode_step.restype = ctypes.c_int
    L.linsimp_decode_chunk.argtypes = [i64, i32, i32, i32, i32, i32, i32, i32, f32] + [vp] * 13 + [vp]
    L.linsimp_decode_chunk.restype = ctypes.c_int
    pa, pg = ctypes.POINTER(AttnDims), ctypes.POINTER(GlrDims)
    L.linsimp_attn_workspace_size.argtypes = [pa, ctypes.c_int]
    L.linsimp_attn_workspace_size.restype = sz
    L.linsimp_attn_fwd.argtypes = [pa] + [vp] * 7 + [vp, sz, vp]
    L.linsimp_attn_fwd.restype = ctypes.c_int
    L.linsimp_attn_bwd.argtypes = [pa] + [vp] * 11 + [vp, sz, vp]
    L.linsimp_attn_bwd.restype = ctypes.c_int
    L.linsimp_attn_step.argtypes = [pa] + [vp] * 7 + [vp, sz, vp]
    L.linsimp_attn_step.restype = ctypes.c_int
    L.linsimp_glr_workspace_size.argtypes = [pg, ctypes.c_int]
    L.linsimp_glr_workspace_size.restype = sz
    L.linsimp_glr_fwd.argtypes = [pg] + [vp] * 8 + [vp, sz, vp]
    L.linsimp_glr_fwd.restype = ctypes.c_int
    L.linsimp_glr_bwd.argtypes = [pg] + [vp] * 13 + [vp, sz, vp]
    L.linsimp_glr_bwd.restype = ctypes.c_int
    L.linsimp_glr_step.argtypes = [pg] + [vp] * 6 + [vp]
    L.linsimp_glr_step.restype = ctypes.c_int
    L.linsimp_timing_enable.argtypes = [ctypes.c_int]
    L.linsimp_timing_enable.restype = ctypes.c_int
    L.linsimp_timing_read.argtypes = [ctypes.c_char_p, ctypes.c_int, ctypes.POINTER(ctypes.c_float),
                                      ctypes.POINTER(ctypes.c_int), ctypes.c_int]
    L.linsimp_timing_read.restype = ctypes.c_int
    L.linsimp_last_error.argtypes = []
    L.linsimp_last_error.restype = ctypes.c_char_p
    L.linsimp_version.argtypes = []
    L.linsimp_version.restype = ctypes.c_int
    po = ctypes.POINTER(HeadOpts)
    L.linsimp_head_saved_size.argtypes = [pd]
    L.linsimp_head_saved_size.restype = sz
    L.linsimp_head_workspace_size.argtypes = [pd, ctypes.c_int]
    L.linsimp_head_workspace_size.restype = sz
    L.linsimp_head_fwd.argtypes = [pd, po] + [vp] * 10 + [sz, vp, sz, vp]
    L.linsimp_head_fwd.restype = ctypes.c_int
    L.linsimp_head_bwd.argtypes = [pd, po] + [vp] * 17 + [vp, sz, vp]
    L.linsimp_head_bwd.restype = ctypes.c_int
    L.linsimp_head_bwd_ex.argtypes = [pd, po] + [vp] * 17 + [i32, vp, sz, vp]
    L.linsimp_head_bwd_ex.restype = ctypes.c_int
    L.linsimp_feature_bank.argtypes = [i32, i32, i32, vp, vp, vp, i32, vp]
    L.linsimp_feature_bank.restype = ctypes.c_int
    _lib = L
    return L


def _check(rc: int):
    if rc != 0:
        raise LinSimpError(rc, lib().linsimp_last_error().decode())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t: Optional[torch.Tensor], name: str):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


try:
    # the raw handle, without the Stream object torch.cuda.current_stream builds
    # (4 us of a 21 us decode step's host time)
    _current_device = torch._C._cuda_getDevice
    _current_raw_stream = torch._C._cuda_getCurrentRawStream
except AttributeError:                                # a torch without these entry points
    _current_device = torch.cuda.current_device

    def _current_raw_stream(device):
        return torch.cuda.current_stream(device).cuda_stream


def _stream():
    return _current_raw_stream(_current_device())


def _expect(pairs):
    """Check (tensor, name, shape, dtype) tuples before their pointers go to
    the C ABI, which sees bare pointers and trusts the sizes it is given: a
    tensor of the wrong shape would be read or written out of bounds.  Shape
    and dtype are checked first, then that every tensor is dense, on a GPU, on
    the first one's device, and that this is the current device (the launch
    stream's).  Returns the tensors' addresses, in order."""
    for t, name, shape, dtype in pairs:
        if t is None:
            raise ValueError(f"{name} is required")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if t.dtype != dtype:
            raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    first = pairs[0][0]
    idx = first.get_device()                          # -1: not a GPU
    ptrs = []
    for t, name, _, _ in pairs:
        if t.get_device() != idx:
            raise ValueError(f"{name} is on {t.device}, expected {first.device}")
        if idx < 0:
            raise ValueError(f"{name} must be a GPU tensor")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        ptrs.append(t.data_ptr())
    if idx != _current_device():
        raise ValueError(f"tensors are on {first.device} but the current device is cuda:{torch.cuda.current_device()}")
    return ptrs


def _layer_shapes(q, v, omega):
    if q.dim() != 4 or v.dim() != 4 or omega.dim() != 3:
        raise ValueError("q, v must be [B, H, n, D|Dv] and omega [H, m, D]")
    B, H, n, D = q.shape
    return B, H, n, D, v.shape[-1], omega.shape[1]


def _layer_inputs(q, k, v, r, u, omega):
    B, H, n, D, Dv, m = _layer_shapes(q, v, omega)
    dt = q.dtype
    return [(q, "q", (B, H, n, D), dt), (k, "k", (B, H, n, D), dt), (v, "v", (B, H, n, Dv), dt),
            (r, "r", (B, H, n, D), dt), (u, "u", (B, H, n, Dv), dt),
            (omega, "omega", (H, m, D), torch.float32)]


def make_dims(B, H, n, D, Dv, m, w, dtype, eps=EPS) -> Dims:
    return Dims(B, H, n, D, Dv, m, w, dtype, eps)


def dims_of(q: torch.Tensor, v: torch.Tensor, omega: torch.Tensor, w: int, eps: float = EPS) -> Dims:
    B, H, n, D = q.shape
    return make_dims(B, H, n, D, v.shape[-1], omega.shape[1], w, _dtype_code(q), eps)


def workspace_size(d: Dims, backward: bool) -> int:
    return int(lib().linsimp_workspace_size(ctypes.byref(d), 1 if backward else 0))


def alloc_workspace(d: Dims, backward: bool, device) -> torch.Tensor:
    nbytes = workspace_size(d, backward)
    if nbytes == 0:
        _check(lib().linsimp_workspace_size(ctypes.byref(d), 1 if backward else 0) or -2)
    ws = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    off = (-ws.data_ptr()) % 256
    return ws[off: off + nbytes]


def fwd(q, k, v, r, u, omega, w, eps=EPS, out=None, stats=None, workspace=None,
        want_stats=True):
    """Forward pass; returns (out, stats).  See linsimp_fwd."""
    chk = _layer_inputs(q, k, v, r, u, omega)
    d = dims_of(q, v, omega, w, eps)
    if out is None:
        out = torch.empty(q.shape[:3] + (v.shape[-1],), dtype=q.dtype, device=q.device)
    if stats is None and want_stats:
        stats = torch.empty(q.shape[:3] + (2,), dtype=torch.float32, device=q.device)
    chk.append((out, "out", q.shape[:3] + (v.shape[-1],), q.dtype))
    if stats is not None:
        chk.append((stats, "stats", q.shape[:3] + (2,), torch.float32))
    ptrs = _expect(chk)
    if stats is None:
        ptrs.append(None)
    if workspace is None:
        workspace = alloc_workspace(d, False, q.device)
    _check(lib().linsimp_fwd(ctypes.byref(d), *ptrs, _ptr(workspace, "workspace"),
                             workspace.numel(), _stream()))
    return out, stats


FWD_STATIC_MAX_BYTES = 64 << 20      # LINSIMP_FWD_STATIC_MAX_BYTES


def fwd_static(q, k, v, r, u, omega, w, eps=EPS, out=None, stats=None, want_stats=True):
    """Forward pass with the library's static scratch instead of a workspace
    (linsimp_fwd_static: nothing is allocated by the library; ``out`` and
    ``stats`` are allocated here unless given); returns (out, stats)."""
    chk = _layer_inputs(q, k, v, r, u, omega)
    d = dims_of(q, v, omega, w, eps)
    if out is None:
        out = torch.empty(q.shape[:3] + (v.shape[-1],), dtype=q.dtype, device=q.device)
    if stats is None and want_stats:
        stats = torch.empty(q.shape[:3] + (2,), dtype=torch.float32, device=q.device)
    chk.append((out, "out", q.shape[:3] + (v.shape[-1],), q.dtype))
    if stats is not None:
        chk.append((stats, "stats", q.shape[:3] + (2,), torch.float32))
    ptrs = _expect(chk)
    if stats is None:
        ptrs.append(None)
    _check(lib().linsimp_fwd_static(ctypes.byref(d), *ptrs, _stream()))
    return out, stats


def bwd(q, k, v, r, u, omega, w, out, stats, dout, eps=EPS, grads=None, workspace=None,
        reuse_states=False):
    """Backward pass; returns (dq, dk, dv, dr, du).  See linsimp_bwd; with
    ``reuse_states`` (linsimp_bwd_ex, LINSIMP_BWD_REUSE_STATES) ``workspace``
    must be the backward-sized workspace the matching fwd call used."""
    chk = _layer_inputs(q, k, v, r, u, omega)
    d = dims_of(q, v, omega, w, eps)
    if grads is None:
        grads = tuple(torch.empty_like(x) for x in (q, k, v, r, u))
    dq, dk, dv, dr, du = grads
    ov = q.shape[:3] + (v.shape[-1],)
    chk += [(out, "out", ov, q.dtype), (stats, "stats", q.shape[:3] + (2,), torch.float32),
            (dout, "dout", ov, q.dtype)]
    chk += [(g, "d" + nm, x.shape, x.dtype) for g, nm, x in zip(grads, "qkvru", (q, k, v, r, u))]
    ptrs = _expect(chk)
    if workspace is None:
        if reuse_states:
            raise ValueError("reuse_states needs the workspace of the matching forward call")
        workspace = alloc_workspace(d, True, q.device)
    _check(lib().linsimp_bwd_ex(ctypes.byref(d), *ptrs, BWD_REUSE_STATES if reuse_states else 0,
                                _ptr(workspace, "workspace"), workspace.numel(), _stream()))
    return dq, dk, dv, dr, du


def timing_enable(on: bool = True):
    """Bracket every library kernel launch with HIP events (see linsimp_timing_enable)."""
    _check(lib().linsimp_timing_enable(1 if on else 0))


def timing_read(max_kernels: int = 64):
    """Per-kernel {name: (total_ms, launches)} since the previous read."""
    names = ctypes.create_string_buffer(4096)
    tot = (ctypes.c_float * max_kernels)()
    cnt = (ctypes.c_int * max_kernels)()
    nk = lib().linsimp_timing_read(names, 4096, tot, cnt, max_kernels)
    if nk < 0:
        _check(nk)
    keys = names.value.decode().split("\n")[:nk]
    return {k: (float(tot[i]), int(cnt[i])) for i, k in enumerate(keys)}


def prefill(k, v, r, u, omega, w, eps=EPS, workspace=None):
    """Decode state after a prefix (k, v, r, u: [S, H, n, *]).  Returns a dict
    with M [S,H,m,Dv], a [S,H,m], rho [S,H] (log2 frame), ring_r, ring_u, pos."""
    S, H, n, D, Dv, m = _layer_shapes(k, v, omega)
    ptrs = _expect([(k, "k", (S, H, n, D), k.dtype), (v, "v", (S, H, n, Dv), k.dtype),
                    (r, "r", (S, H, n, D), k.dtype), (u, "u", (S, H, n, Dv), k.dtype),
                    (omega, "omega", (H, m, D), torch.float32)])
    d = make_dims(S, H, n, D, Dv, m, w, _dtype_code(k), eps)
    dev = k.device
    st = {"M": torch.empty(S, H, m, Dv, dtype=torch.float32, device=dev),
          "a": torch.empty(S, H, m, dtype=torch.float32, device=dev),
          "rho": torch.empty(S, H, dtype=torch.float32, device=dev),
          "ring_r": torch.empty(S, H, w, D, dtype=k.dtype, device=dev),
          "ring_u": torch.empty(S, H, w, Dv, dtype=k.dtype, device=dev),
          "pos": torch.empty(S, dtype=torch.int64, device=dev)}
    if workspace is None:
        workspace = alloc_workspace(d, False, dev)
    _check(lib().linsimp_prefill(ctypes.byref(d), *ptrs, *[t.data_ptr() for t in st.values()],
                                 _ptr(workspace, "workspace"), workspace.numel(), _stream()))
    return st


def _decode_checks(state, q, k, v, r, u, omega, w, out, tok):
    """Shapes of a decode call: tok is () for one token, (T,) for a chunk."""
    if q.dim() != 3 + len(tok) or omega.dim() != 3:
        raise ValueError("q must be [S, H, *tok, D] and omega [H, m, D]")
    S, H, D = q.shape[0], q.shape[1], q.shape[-1]
    Dv, m, dt = v.shape[-1], omega.shape[1], q.dtype
    f32 = torch.float32
    sD, sV = (S, H, *tok, D), (S, H, *tok, Dv)
    ptrs = _expect([(q, "q", sD, dt), (k, "k", sD, dt), (v, "v", sV, dt), (r, "r", sD, dt), (u, "u", sV, dt),
                    (omega, "omega", (H, m, D), f32), (state["M"], "M", (S, H, m, Dv), f32),
                    (state["a"], "a", (S, H, m), f32), (state["rho"], "rho", (S, H), f32),
                    (state["ring_r"], "ring_r", (S, H, w, D), dt), (state["ring_u"], "ring_u", (S, H, w, Dv), dt),
                    (state["pos"], "pos", (S,), torch.int64), (out, "out", sV, dt)])
    return S, H, D, Dv, m, ptrs


def decode_step(state, q, k, v, r, u, omega, w, eps=EPS, out=None):
    """One decode step for S sequences (q, k, v, r, u: [S, H, *]); updates
    ``state`` in place and returns out [S, H, Dv]."""
    if out is None:
        out = q.new_empty(q.shape[:2] + (v.shape[-1],))
    S, H, D, Dv, m, ptrs = _decode_checks(state, q, k, v, r, u, omega, w, out, ())
    _check(lib().linsimp_decode_step(S, H, D, Dv, m, w, _dtype_code(q), eps, *ptrs, _stream()))
    return out


def decode_chunk(state, q, k, v, r, u, omega, w, eps=EPS, out=None):
    """T consecutive decode steps for S sequences (q, k, v, r, u: [S, H, T, *]);
    updates ``state`` in place and returns out [S, H, T, Dv]."""
    if out is None:
        out = torch.empty(q.shape[:3] + (v.shape[-1],), dtype=q.dtype, device=q.device)
    T = q.shape[2]
    S, H, D, Dv, m, ptrs = _decode_checks(state, q, k, v, r, u, omega, w, out, (T,))
    _check(lib().linsimp_decode_chunk(S, H, T, D, Dv, m, w, _dtype_code(q), eps, *ptrs, _stream()))
    return out


# ---------------------------------------------------------------------------
# Full head (include/linsimp_head.h)
# ---------------------------------------------------------------------------

def _aligned_bytes(nbytes: int, device) -> torch.Tensor:
    buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 256
    return buf[off: off + nbytes]


def head_opts(gate_kind=GATE_HEAD, norm_eps=NORM_EPS, rms_eps=RMS_EPS) -> HeadOpts:
    return HeadOpts(norm_eps, rms_eps, gate_kind)


def _gate_kind(gate: torch.Tensor, v: torch.Tensor) -> int:
    return GATE_CHANNEL if gate.dim() == 4 else GATE_HEAD


def _head_params(q, v, tau, gate):
    H = q.shape[1]
    gshape, gdt = ((q.shape[:3] + (v.shape[-1],), q.dtype) if gate.dim() == 4 else ((H,), torch.float32))
    return [(tau, "tau", (H,), torch.float32), (gate, "gate", gshape, gdt)]


def head_fwd(q, k, v, r, u, omega, w, tau, gate, eps=EPS, norm_eps=NORM_EPS, rms_eps=RMS_EPS,
             y=None, saved=None, workspace=None):
    """Forward of one full head; returns (y, saved).  ``gate`` is gamma [H]
    float32 (per-head gate) or logits [B, H, n, Dv] (channel-wise gate).
    See linsimp_head_fwd."""
    d = dims_of(q, v, omega, w, eps)
    o = head_opts(_gate_kind(gate, v), norm_eps, rms_eps)
    L = lib()
    if y is None:
        y = torch.empty(q.shape[:3] + (v.shape[-1],), dtype=q.dtype, device=q.device)
    _expect(_layer_inputs(q, k, v, r, u, omega) + _head_params(q, v, tau, gate)
            + [(y, "y", q.shape[:3] + (v.shape[-1],), q.dtype)])
    if saved is None:
        nb = int(L.linsimp_head_saved_size(ctypes.byref(d)))
        if nb == 0:
            _check(-2)
        saved = _aligned_bytes(nb, q.device)
    if workspace is None:
        nb = int(L.linsimp_head_workspace_size(ctypes.byref(d), 0))
        if nb == 0:
            _check(-2)
        workspace = _aligned_bytes(nb, q.device)
    _check(L.linsimp_head_fwd(ctypes.byref(d), ctypes.byref(o), _ptr(q, "q"), _ptr(k, "k"),
                              _ptr(v, "v"), _ptr(r, "r"), _ptr(u, "u"), _ptr(omega, "omega"),
                              _ptr(tau, "tau"), _ptr(gate, "gate"), _ptr(y, "y"),
                              _ptr(saved, "saved"), saved.numel(), _ptr(workspace, "workspace"),
                              workspace.numel(), _stream()))
    return y, saved


def head_bwd(q, k, v, r, u, omega, w, tau, gate, saved, dy, eps=EPS, norm_eps=NORM_EPS,
             rms_eps=RMS_EPS, workspace=None, reuse_states=False):
    """Backward of one full head; returns (dq, dk, dv, dr, du, dtau, dgate).
    See linsimp_head_bwd; with ``reuse_states`` (linsimp_head_bwd_ex)
    ``workspace`` must be the backward-sized one the matching head_fwd used."""
    d = dims_of(q, v, omega, w, eps)
    o = head_opts(_gate_kind(gate, v), norm_eps, rms_eps)
    L = lib()
    _expect(_layer_inputs(q, k, v, r, u, omega) + _head_params(q, v, tau, gate)
            + [(dy, "dy", q.shape[:3] + (v.shape[-1],), q.dtype)])
    grads = [torch.empty_like(x) for x in (q, k, v, r, u)]
    dtau = torch.empty_like(tau)
    dgate = torch.empty_like(gate)
    if workspace is None:
        if reuse_states:
            raise ValueError("reuse_states needs the workspace of the matching head_fwd call")
        nb = int(L.linsimp_head_workspace_size(ctypes.byref(d), 1))
        if nb == 0:
            _check(-2)
        workspace = _aligned_bytes(nb, q.device)
    _check(L.linsimp_head_bwd_ex(ctypes.byref(d), ctypes.byref(o), _ptr(q, "q"), _ptr(k, "k"),
                                 _ptr(v, "v"), _ptr(r, "r"), _ptr(u, "u"), _ptr(omega, "omega"),
                                 _ptr(tau, "tau"), _ptr(gate, "gate"), _ptr(saved, "saved"),
                                 _ptr(dy, "dy"), *[_ptr(g, "grad") for g in grads],
                                 _ptr(dtau, "dtau"), _ptr(dgate, "dgate"),
                                 BWD_REUSE_STATES if reuse_states else 0,
                                 _ptr(workspace, "workspace"), workspace.numel(), _stream()))
    return (*grads, dtau, dgate)


# ---------------------------------------------------------------------------
# Orthogonal random-feature bank (include/linsimp_bank.h)
# ---------------------------------------------------------------------------

def feature_bank(gauss, radii, m, sign_correct=True, omega=None):
    """Bank [H, m, D] float32 from draws gauss [H, nb, D, D] and radii
    [H, nb, D] (float32, on the GPU).  See linsimp_feature_bank."""
    H, nb, D, _ = gauss.shape
    if gauss.dtype != torch.float32 or radii.dtype != torch.float32:
        raise TypeError("gauss and radii must be float32")
    if radii.shape != (H, nb, D) or nb != (m + D - 1) // D:
        raise ValueError("gauss must be [H, ceil(m/D), D, D] and radii [H, ceil(m/D), D]")
    if omega is None:
        omega = torch.empty(H, m, D, dtype=torch.float32, device=gauss.device)
    _check(lib().linsimp_feature_bank(H, m, D, _ptr(gauss, "gauss"), _ptr(radii, "radii"),
                                      _ptr(omega, "omega"), 1 if sign_correct else 0, _stream()))
    return omega


# ---------------------------------------------------------------------------
# Softmax attention and the gated linear recurrence (include/linsimp.h)
# ---------------------------------------------------------------------------

def alloc_bytes(nbytes: int, device) -> torch.Tensor:
    """A 256-byte aligned workspace of ``nbytes`` bytes."""
    return _aligned_bytes(nbytes, device)


def attn_dims(q, k, causal=True, window=0, scale=None) -> AttnDims:
    """Dims of an attention call from q [B, H, nq, D] and k [B, Hkv, nk, D]."""
    if q.dim() != 4 or k.dim() != 4:
        raise ValueError("q must be [B, H, nq, D] and k [B, Hkv, nk, D]")
    B, H, nq, D = q.shape
    return AttnDims(B, H, k.shape[1], nq, k.shape[2], window, D, _dtype_code(q), 1 if causal else 0,
                    D ** -0.5 if scale is None else scale)


def glr_dims(q, scale=None) -> GlrDims:
    """Dims of a recurrence call from q [B, H, n, D] (or [B, H, D]: one row)."""
    if q.dim() not in (3, 4):
        raise ValueError("q must be [B, H, n, D] or [B, H, D]")
    B, H, D = q.shape[0], q.shape[1], q.shape[-1]
    return GlrDims(B, H, q.shape[2] if q.dim() == 4 else 1, D, _dtype_code(q), D ** -0.5 if scale is None else scale)


def attn_workspace_size(d: AttnDims, backward: bool) -> int:
    return int(lib().linsimp_attn_workspace_size(ctypes.byref(d), 1 if backward else 0))


def glr_workspace_size(d: GlrDims, backward: bool) -> int:
    return int(lib().linsimp_glr_workspace_size(ctypes.byref(d), 1 if backward else 0))


def _mixer_workspace(workspace, nbytes, device):
    """The caller's workspace (the library checks its size, and the dims), or a new
    one of ``nbytes`` (None beside a caller's: the size costs a call)."""
    if workspace is None:
        if nbytes == 0:
            _check(-2)                                 # the message of the refused dims
        return alloc_bytes(nbytes, device)
    if workspace.get_device() != device.index:
        raise ValueError(f"workspace is on {workspace.device}, expected {device}")
    return workspace


def _with_optional(pairs, optional):
    """_expect over the required (tensor, name, shape, dtype) and those of
    ``optional`` that are given; the addresses of both, None for the others."""
    ptrs = _expect(pairs + [p for p in optional if p[0] is not None])
    it = iter(ptrs[len(pairs):])
    return ptrs[:len(pairs)], [next(it) if p[0] is not None else None for p in optional]


def _attn_inputs(q, k, v, d):
    return [(q, "q", (d.B, d.H, d.nq, d.D), q.dtype), (k, "k", (d.B, d.Hkv, d.nk, d.D), q.dtype),
            (v, "v", (d.B, d.Hkv, d.nk, d.D), q.dtype)]


def _attn_lens(lens_q, lens_k, B):
    return [(lens_q, "lens_q", (B,), torch.int32), (lens_k, "lens_k", (B,), torch.int32)]


def attn_fwd(q, k, v, causal=True, window=0, scale=None, lens_q=None, lens_k=None, out=None, lse=None,
             want_lse=True, workspace=None):
    """Softmax attention of q [B, H, nq, D] over k, v [B, Hkv, nk, D]; returns
    (out, lse).  See linsimp_attn_fwd."""
    d = attn_dims(q, k, causal, window, scale)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if lse is None and want_lse:
        lse = torch.empty(q.shape[:3], dtype=torch.float32, device=q.device)
    ptrs, (pq, pk, pl) = _with_optional(
        _attn_inputs(q, k, v, d) + [(out, "out", q.shape, q.dtype)],
        _attn_lens(lens_q, lens_k, d.B) + [(lse, "lse", q.shape[:3], torch.float32)])
    nbytes = attn_workspace_size(d, False) if workspace is None else None
    workspace = _mixer_workspace(workspace, nbytes, q.device)
    _check(lib().linsimp_attn_fwd(ctypes.byref(d), *ptrs[:3], pq, pk, ptrs[3], pl, _ptr(workspace, "workspace"),
                                  workspace.numel(), _stream()))
    return out, lse


def attn_bwd(q, k, v, out, lse, dout, causal=True, window=0, scale=None, lens_q=None, lens_k=None, grads=None,
             workspace=None):
    """Backward of attn_fwd from what it returned; returns (dq, dk, dv).  See
    linsimp_attn_bwd."""
    d = attn_dims(q, k, causal, window, scale)
    if grads is None:
        grads = tuple(torch.empty_like(x, memory_format=torch.contiguous_format) for x in (q, k, v))
    ptrs, (pq, pk) = _with_optional(
        _attn_inputs(q, k, v, d)
        + [(out, "out", q.shape, q.dtype), (lse, "lse", q.shape[:3], torch.float32), (dout, "dout", q.shape, q.dtype)]
        + [(g, "d" + nm, x.shape, x.dtype) for g, nm, x in zip(grads, "qkv", (q, k, v))],
        _attn_lens(lens_q, lens_k, d.B))
    nbytes = attn_workspace_size(d, True) if workspace is None else None
    workspace = _mixer_workspace(workspace, nbytes, q.device)
    _check(lib().linsimp_attn_bwd(ctypes.byref(d), *ptrs[:3], pq, pk, *ptrs[3:], _ptr(workspace, "workspace"),
                                  workspace.numel(), _stream()))
    return tuple(grads)


def attn_step(kcache, vcache, pos, q, k, v, scale=None, out=None, workspace=None):
    """One decode step: token pos[b] (q [B, H, D], k, v [B, Hkv, D]) enters the ring
    caches [B, Hkv, slots, D] in place; returns out [B, H, D].  See
    linsimp_attn_step."""
    if q.dim() != 3 or kcache.dim() != 4:
        raise ValueError("q must be [B, H, D] and kcache [B, Hkv, slots, D]")
    B, H, D = q.shape
    Hkv, cap = kcache.shape[1], kcache.shape[2]
    d = AttnDims(B, H, Hkv, 1, cap, 0, D, _dtype_code(q), 1, D ** -0.5 if scale is None else scale)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    dt = q.dtype
    ptrs = _expect([(q, "q", (B, H, D), dt), (k, "k", (B, Hkv, D), dt), (v, "v", (B, Hkv, D), dt),
                    (kcache, "kcache", (B, Hkv, cap, D), dt), (vcache, "vcache", (B, Hkv, cap, D), dt),
                    (pos, "pos", (B,), torch.int64), (out, "out", (B, H, D), dt)])
    nbytes = attn_workspace_size(d, False) if workspace is None else None
    workspace = _mixer_workspace(workspace, nbytes, q.device)
    _check(lib().linsimp_attn_step(ctypes.byref(d), *ptrs, _ptr(workspace, "workspace"), workspace.numel(),
                                   _stream()))
    return out


def _glr_inputs(q, k, v, g):
    return [(x, nm, q.shape, q.dtype) for x, nm in ((q, "q"), (k, "k"), (v, "v"), (g, "g"))]


def glr_fwd(q, k, v, g, s0=None, lens=None, scale=None, out=None, s1=None, want_state=True, workspace=None):
    """Gated linear recurrence over q, k, v, g [B, H, n, D]; returns (out, s1), s1
    the state [B, H, D, D] after the last row (None without ``want_state``).
    See linsimp_glr_fwd."""
    d = glr_dims(q, scale)
    st = (d.B, d.H, d.D, d.D)
    if q.dim() != 4:
        raise ValueError("q must be [B, H, n, D]")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if s1 is None and want_state:
        s1 = torch.empty(st, dtype=torch.float32, device=q.device)
    ptrs, (p0, pl, p1) = _with_optional(
        _glr_inputs(q, k, v, g) + [(out, "out", q.shape, q.dtype)],
        [(s0, "s0", st, torch.float32), (lens, "lens", (d.B,), torch.int32), (s1, "s1", st, torch.float32)])
    nbytes = glr_workspace_size(d, False) if workspace is None else None
    workspace = _mixer_workspace(workspace, nbytes, q.device)
    _check(lib().linsimp_glr_fwd(ctypes.byref(d), *ptrs[:4], p0, pl, ptrs[4], p1, _ptr(workspace, "workspace"),
                                 workspace.numel(), _stream()))
    return out, s1


def glr_bwd(q, k, v, g, dout, s0=None, lens=None, ds1=None, scale=None, grads=None, want_ds0=None, workspace=None):
    """Backward of glr_fwd; returns (dq, dk, dv, dg, ds0), ds0 None unless there is
    an s0 (or ``want_ds0``).  See linsimp_glr_bwd."""
    d = glr_dims(q, scale)
    st = (d.B, d.H, d.D, d.D)
    if q.dim() != 4:
        raise ValueError("q must be [B, H, n, D]")
    if grads is None:
        grads = tuple(torch.empty_like(x, memory_format=torch.contiguous_format) for x in (q, k, v, g))
    ds0 = None
    if want_ds0 if want_ds0 is not None else s0 is not None:
        ds0 = torch.empty(st, dtype=torch.float32, device=q.device)
    ptrs, (p0, pl, p1, pd) = _with_optional(
        _glr_inputs(q, k, v, g) + [(dout, "dout", q.shape, q.dtype)]
        + [(x, "d" + nm, q.shape, q.dtype) for x, nm in zip(grads, "qkvg")],
        [(s0, "s0", st, torch.float32), (lens, "lens", (d.B,), torch.int32), (ds1, "ds1", st, torch.float32),
         (ds0, "ds0", st, torch.float32)])
    nbytes = glr_workspace_size(d, True) if workspace is None else None
    workspace = _mixer_workspace(workspace, nbytes, q.device)
    _check(lib().linsimp_glr_bwd(ctypes.byref(d), *ptrs[:4], p0, pl, ptrs[4], p1, *ptrs[5:], pd,
                                 _ptr(workspace, "workspace"), workspace.numel(), _stream()))
    return (*grads, ds0)


def glr_step(state, q, k, v, g, scale=None, out=None):
    """One decode step (q, k, v, g: [B, H, D]); updates ``state`` [B, H, D, D] in
    place and returns out [B, H, D].  See linsimp_glr_step."""
    if q.dim() != 3:
        raise ValueError("q must be [B, H, D]")
    d = glr_dims(q, scale)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    ptrs = _expect(_glr_inputs(q, k, v, g) + [(state, "state", (d.B, d.H, d.D, d.D), torch.float32),
                                             (out, "out", q.shape, q.dtype)])
    _check(lib().linsimp_glr_step(ctypes.byref(d), *ptrs, _stream()))
    return out
