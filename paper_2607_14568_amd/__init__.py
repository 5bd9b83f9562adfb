"""Gated delta-rule prefill and decode on MI355X (gfx950).

A thin ctypes binding over ``libgdn.so`` (C ABI in ``include/gdn.h``).  The
functions carry the C names and only marshal arguments: every step of the
computation runs in the library's HIP kernels.  PyTorch supplies device memory
and the current stream.  There is no CPU fallback: if the library is not built
or no GPU is present, calls raise.
"""
from __future__ import annotations

import ctypes
import os

import torch

__all__ = [
    "GDN_F32", "GDN_BF16", "GdnError", "lib", "gdn_version", "gdn_status_string",
    "gdn_chunk_prefill_workspace_bytes", "gdn_chunk_prefill_workspace_bytes_ex", "gdn_chunk_prefill",
    "gdn_decode_step", "gdn_chunk_prefill_plan", "gdn_chunk_prefill_snapshots",
    "GDN_PLAN_SEQUENTIAL", "GDN_PLAN_SEGMENTED", "GDN_PLAN_WIDE",
    "gdn_chunk_prefill_grouped", "gdn_decode_step_grouped", "gdn_chunk_prefill_ex", "gdn_decode_step_ex",
    "GDN_QK_L2NORM", "GDN_GATE_LOGITS", "gdn_attention_prefill", "gdn_chunk_prefill_snapshots_ex",
    "gdn_workspace_status", "GDN_ERR_WAIT", "GDN_TEST_WITHHOLD",
    "GDN_E4M3", "GDN_ROPE_INTERLEAVED", "gdn_qk_norm_rope", "gdn_kv_append", "gdn_attention_paged",
    "gdn_attention_paged_workspace_bytes",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgdn.so")

GDN_F32, GDN_BF16, GDN_E4M3 = 0, 1, 2
GDN_QK_L2NORM, GDN_GATE_LOGITS = 1, 2
GDN_PLAN_SEQUENTIAL, GDN_PLAN_SEGMENTED, GDN_PLAN_WIDE = 16, 32, 64
GDN_TEST_WITHHOLD = 256
GDN_ROPE_INTERLEAVED = 512
GDN_ERR_WAIT = 5
_IO = {torch.float32: GDN_F32, torch.bfloat16: GDN_BF16}
_CACHE = {torch.bfloat16: GDN_BF16, torch.float8_e4m3fn: GDN_E4M3}
_lib = None


class GdnError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("%s: %s" % (gdn_status_string(status), message))
        self.status = status


def lib():
    """The loaded ``libgdn.so`` (ctypes.CDLL) with argument types declared."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libgdn.so is not built (%s); run __graft_entry__.build()" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        P, I, F, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        L.gdn_version.restype = I
        L.gdn_status_string.argtypes = [I]
        L.gdn_status_string.restype = ctypes.c_char_p
        L.gdn_last_error_message.restype = ctypes.c_char_p
        L.gdn_chunk_prefill_workspace_bytes.argtypes = [I, I, I, I, I, I, I, I]
        L.gdn_chunk_prefill_workspace_bytes.restype = S
        L.gdn_chunk_prefill_workspace_bytes_ex.argtypes = [I] * 10
        L.gdn_chunk_prefill_workspace_bytes_ex.restype = S
        L.gdn_chunk_prefill.argtypes = [P, P, P, P, P, P, P, P, I, I, I, I, I, I, P, I, I, F, P, S, P]
        L.gdn_chunk_prefill.restype = I
        L.gdn_chunk_prefill_grouped.argtypes = [P, P, P, P, P, P, P, P, I, I, I, I, I, I, I, P, I, I, F, P, S, P]
        L.gdn_chunk_prefill_grouped.restype = I
        L.gdn_chunk_prefill_ex.argtypes = [P, P, P, P, P, P, P, P, I, I, I, I, I, I, I, P, I, I, F, I, I, P, S, P]
        L.gdn_chunk_prefill_ex.restype = I
        L.gdn_chunk_prefill_snapshots.argtypes = [P, P, P, P, P, P, P, P, I, I, I, I, I, I, P, I, I, F, I, P, P, S,
                                                  P]
        L.gdn_chunk_prefill_snapshots.restype = I
        L.gdn_chunk_prefill_snapshots_ex.argtypes = [P, P, P, P, P, P, P, P, I, I, I, I, I, I, I, P, I, I, F, I, I, P, P,
                                                     S, P]
        L.gdn_chunk_prefill_snapshots_ex.restype = I
        L.gdn_chunk_prefill_noalloc.argtypes = [P, P, P, P, P, P, P, P, I, I, I, I, I, I, I, P, I, I, F, I, I, P]
        L.gdn_chunk_prefill_noalloc.restype = I
        L.gdn_chunk_prefill_plan.argtypes = [I, I, I, I, I, I, I, I, I, S, P, ctypes.POINTER(I)]
        L.gdn_chunk_prefill_plan.restype = I
        L.gdn_decode_step.argtypes = [P, P, P, P, P, P, P, I, I, I, I, I, F, P]
        L.gdn_decode_step.restype = I
        L.gdn_decode_step_grouped.argtypes = [P, P, P, P, P, P, P, I, I, I, I, I, I, F, P]
        L.gdn_decode_step_grouped.restype = I
        L.gdn_decode_step_ex.argtypes = [P, P, P, P, P, P, P, I, I, I, I, I, I, F, I, P]
        L.gdn_decode_step_ex.restype = I
        L.gdn_attention_prefill.argtypes = [P, P, P, P, I, I, I, I, I, P, I, I, F, P]
        L.gdn_attention_prefill.restype = I
        LL = ctypes.c_longlong
        L.gdn_qk_norm_rope.argtypes = [P, P, P, P, I, I, I, I, I, LL, LL, P, P, F, P, I, P, P, I, I, I, P]
        L.gdn_qk_norm_rope.restype = I
        L.gdn_kv_append.argtypes = [P] * 10 + [I] * 8 + [LL] * 3 + [P, P, F, P, I, P, I, I, I, I, P]
        L.gdn_kv_append.restype = I
        L.gdn_attention_paged_workspace_bytes.argtypes = [I] * 8
        L.gdn_attention_paged_workspace_bytes.restype = S
        L.gdn_attention_paged.argtypes = [P] * 8 + [I] * 8 + [P, I, I, I, F, P, S, P]
        L.gdn_attention_paged.restype = I
        L.gdn_workspace_status.argtypes = [P, S, P]
        L.gdn_workspace_status.restype = I
        _lib = L
    return _lib


def gdn_version() -> int:
    return int(lib().gdn_version())


def gdn_status_string(status: int) -> str:
    return lib().gdn_status_string(int(status)).decode()


def _check(status):
    if status != 0:
        raise GdnError(status, lib().gdn_last_error_message().decode())


def gdn_workspace_status(workspace=None, device=None):
    """Waits for the current stream and raises GdnError(GDN_ERR_WAIT) if a one-launch prefill on ``workspace``
    (a uint8 CUDA tensor; None: the scratch of ``gdn_chunk_prefill_noalloc``) gave up waiting for its chunk terms
    since the last check (the word is then cleared)."""
    if workspace is None:
        dev = torch.device("cuda", torch.cuda.current_device() if device is None else device)
        _check(lib().gdn_workspace_status(None, 0, _stream(dev)))
    else:
        _dev(workspace, "workspace")
        _check(lib().gdn_workspace_status(_ptr(workspace), workspace.numel() * workspace.element_size(),
                                          _stream(workspace.device)))


def gdn_chunk_prefill_workspace_bytes(B, T, H, dk, dv, chunk=64, n_seqs=0, io_dtype=GDN_BF16) -> int:
    return int(lib().gdn_chunk_prefill_workspace_bytes(B, T, H, dk, dv, chunk, n_seqs, io_dtype))


def gdn_chunk_prefill_workspace_bytes_ex(B, T, H, dk, dv, chunk=64, n_seqs=0, io_dtype=GDN_BF16, flags=0,
                                         segments=0) -> int:
    return int(lib().gdn_chunk_prefill_workspace_bytes_ex(B, T, H, dk, dv, chunk, n_seqs, io_dtype, int(flags),
                                                          int(segments)))


def gdn_chunk_prefill_plan(B, T, H, dk, dv, n_seqs=0, io_dtype=GDN_BF16, flags=0, segments=0,
                           workspace_bytes=None, device=None):
    """``(form, segments)`` a prefill of these sizes would take on ``device`` (form: a GDN_PLAN_* bit).

    ``workspace_bytes`` defaults to what ``gdn_chunk_prefill_workspace_bytes_ex`` gives.
    """
    if workspace_bytes is None:
        workspace_bytes = gdn_chunk_prefill_workspace_bytes_ex(B, T, H, dk, dv, 64, n_seqs, io_dtype, flags, segments)
    form = ctypes.c_int(0)
    stream = _stream(torch.device("cuda", torch.cuda.current_device() if device is None else device))
    n = int(lib().gdn_chunk_prefill_plan(B, T, H, dk, dv, n_seqs, io_dtype, int(flags), int(segments),
                                         int(workspace_bytes), stream, ctypes.byref(form)))
    return int(form.value), n


def _dev(t, name, dtype=None):
    if isinstance(t, torch.Tensor) and t.is_cuda and (dtype is None or t.dtype is dtype) and t.is_contiguous():
        return t
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return t


def _ptr(t):
    return None if t is None else t.data_ptr()   # (ctypes converts the integer by the declared argument type)


# The raw handle of the current stream: a call of a few microseconds' work would otherwise spend a tenth of them on
# building a torch.cuda.Stream object around it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device):
    if _raw_stream is not None and device.index is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _prefill_args(q, k, v, g, beta, S0, chunk, cu_seqlens, o, S_T, store_state, workspace, grouped=False, flags=0,
                  segments=0, with_workspace=True):
    if q.dtype not in _IO:
        raise TypeError("q must be float32 or bfloat16")
    io = _IO[q.dtype]
    for name, t in (("q", q), ("k", k), ("v", v)):
        _dev(t, name, q.dtype)
    _dev(g, "g", torch.float32)
    _dev(beta, "beta", torch.float32)
    B, T, HK, dk = q.shape
    H = v.shape[2] if grouped else HK
    dv = v.shape[-1]
    if k.shape != q.shape or tuple(v.shape[:3]) != (B, T, H) or tuple(g.shape) != (B, T, H) \
            or beta.shape != g.shape:
        raise ValueError("inconsistent shapes q%s k%s v%s g%s beta%s" % (
            tuple(q.shape), tuple(k.shape), tuple(v.shape), tuple(g.shape), tuple(beta.shape)))
    n_seqs = 0
    if cu_seqlens is not None:
        _dev(cu_seqlens, "cu_seqlens", torch.int32)
        n_seqs = cu_seqlens.numel() - 1
    n = n_seqs if n_seqs else B
    if S0 is not None:
        _dev(S0, "S0", torch.float32)
        if tuple(S0.shape) != (n, H, dv, dk):
            raise ValueError("S0 must be [%d,%d,%d,%d]" % (n, H, dv, dk))
    if o is None:
        o = torch.empty_like(v)
    else:
        _dev(o, "o", q.dtype)
    if store_state and S_T is None:
        S_T = torch.empty((n, H, dv, dk), device=q.device, dtype=torch.float32)
    elif S_T is not None:
        _dev(S_T, "S_T", torch.float32)
    if not with_workspace:
        return dict(io=io, B=B, T=T, H=H, HK=HK, dk=dk, dv=dv, n=n, n_seqs=n_seqs, o=o, S_T=S_T)
    need = gdn_chunk_prefill_workspace_bytes_ex(B, T, H, dk, dv, chunk, n_seqs, io, flags, segments)
    if workspace is None:
        workspace = torch.empty(max(need, 1), device=q.device, dtype=torch.uint8)
    return dict(io=io, B=B, T=T, H=H, HK=HK, dk=dk, dv=dv, n=n, n_seqs=n_seqs, o=o, S_T=S_T, workspace=workspace)


def gdn_chunk_prefill(q, k, v, g, beta, S0=None, *, chunk=64, cu_seqlens=None, scale=1.0,
                      o=None, S_T=None, store_state=True, workspace=None):
    """Chunked prefill; see ``gdn_chunk_prefill`` in include/gdn.h.

    q,k [B,T,H,dk] and v [B,T,H,dv] (fp32 or bf16, same dtype); g, beta [B,T,H]
    fp32; S0 [n,H,dv,dk] fp32 or None.  Ragged: B == 1 and ``cu_seqlens`` an
    int32 CUDA tensor [n+1].  Returns ``(o, S_T)`` (S_T is None when
    ``store_state`` is False).  ``S_T`` may be passed (also ``S_T is S0``).
    """
    a = _prefill_args(q, k, v, g, beta, S0, chunk, cu_seqlens, o, S_T, store_state, workspace)
    _check(lib().gdn_chunk_prefill(
        _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(S0), _ptr(a["o"]), _ptr(a["S_T"]),
        a["B"], a["T"], a["H"], a["dk"], a["dv"], chunk, _ptr(cu_seqlens), a["n_seqs"], a["io"], float(scale),
        _ptr(a["workspace"]), a["workspace"].numel(), _stream(q.device)))
    return a["o"], a["S_T"]


def gdn_chunk_prefill_grouped(q, k, v, g, beta, S0=None, *, chunk=64, cu_seqlens=None, scale=1.0,
                              o=None, S_T=None, store_state=True, workspace=None):
    """Prefill with grouped key heads; see ``gdn_chunk_prefill_grouped`` in include/gdn.h.

    q,k [B,T,H_k,dk]; v [B,T,H,dv]; g, beta [B,T,H]; value head h reads key head
    h // (H // H_k).  Otherwise as ``gdn_chunk_prefill``.
    """
    a = _prefill_args(q, k, v, g, beta, S0, chunk, cu_seqlens, o, S_T, store_state, workspace, grouped=True)
    _check(lib().gdn_chunk_prefill_grouped(
        _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(S0), _ptr(a["o"]), _ptr(a["S_T"]),
        a["B"], a["T"], a["H"], a["HK"], a["dk"], a["dv"], chunk, _ptr(cu_seqlens), a["n_seqs"], a["io"],
        float(scale), _ptr(a["workspace"]), a["workspace"].numel(), _stream(q.device)))
    return a["o"], a["S_T"]


def gdn_chunk_prefill_ex(q, k, v, g, beta, S0=None, *, flags=0, segments=0, chunk=64, cu_seqlens=None, scale=1.0,
                         o=None, S_T=None, store_state=True, workspace=None):
    """Prefill with in-kernel input transforms and a per-call plan; see ``gdn_chunk_prefill_ex`` in include/gdn.h.

    Shapes as ``gdn_chunk_prefill_grouped``.  ``flags``: GDN_QK_L2NORM (q, k taken
    unnormalised) and/or GDN_GATE_LOGITS (``g``, ``beta`` hold the logits a, b), and at
    most one of GDN_PLAN_SEQUENTIAL, GDN_PLAN_SEGMENTED, GDN_PLAN_WIDE; ``segments``
    the segments per sequence of a segmented plan (0: the plan's own count).
    """
    a = _prefill_args(q, k, v, g, beta, S0, chunk, cu_seqlens, o, S_T, store_state, workspace, grouped=True,
                      flags=flags, segments=segments)
    _check(lib().gdn_chunk_prefill_ex(
        _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(S0), _ptr(a["o"]), _ptr(a["S_T"]),
        a["B"], a["T"], a["H"], a["HK"], a["dk"], a["dv"], chunk, _ptr(cu_seqlens), a["n_seqs"], a["io"],
        float(scale), int(flags), int(segments), _ptr(a["workspace"]), a["workspace"].numel(), _stream(q.device)))
    return a["o"], a["S_T"]


GDN_NOALLOC_SCRATCH_BYTES = 64 << 20


def gdn_chunk_prefill_noalloc(q, k, v, g, beta, S0=None, *, flags=0, segments=0, chunk=64, cu_seqlens=None,
                              scale=1.0, o=None, S_T=None, store_state=True):
    """``gdn_chunk_prefill_ex`` on the library's own per-device scratch (no workspace, no device
    allocation inside the call); see ``gdn_chunk_prefill_noalloc`` in include/gdn.h.  Pass ``o``
    (and ``S_T``, or ``store_state=False``) to allocate nothing here either."""
    a = _prefill_args(q, k, v, g, beta, S0, chunk, cu_seqlens, o, S_T, store_state, None, grouped=True,
                      flags=flags, segments=segments, with_workspace=False)
    _check(lib().gdn_chunk_prefill_noalloc(
        _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(S0), _ptr(a["o"]), _ptr(a["S_T"]),
        a["B"], a["T"], a["H"], a["HK"], a["dk"], a["dv"], chunk, _ptr(cu_seqlens), a["n_seqs"], a["io"],
        float(scale), int(flags), int(segments), _stream(q.device)))
    return a["o"], a["S_T"]


def gdn_chunk_prefill_snapshots(q, k, v, g, beta, S0=None, *, snap_every, chunk=64, cu_seqlens=None, scale=1.0,
                                o=None, S_T=None, snaps=None, store_state=True, workspace=None):
    """Prefill that also returns state snapshots; see ``gdn_chunk_prefill_snapshots`` in include/gdn.h.

    Returns ``(o, S_T, snaps)``; ``snaps`` is [n, (T-1) // (snap_every*chunk), H, dv, dk] fp32
    (allocated zero-filled when not given; entries past a sequence's last snapshot keep their values).
    """
    a = _prefill_args(q, k, v, g, beta, S0, chunk, cu_seqlens, o, S_T, store_state, workspace)
    n_snap = max(0, (a["T"] - 1) // (int(snap_every) * chunk)) if snap_every >= 1 else 0
    shape = (a["n"], n_snap, a["H"], a["dv"], a["dk"])
    if snaps is None:
        snaps = torch.zeros(shape, device=q.device, dtype=torch.float32)
    else:
        _dev(snaps, "snaps", torch.float32)
        if tuple(snaps.shape) != shape:
            raise ValueError("snaps must be %s" % (shape,))
    _check(lib().gdn_chunk_prefill_snapshots(
        _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(S0), _ptr(a["o"]), _ptr(a["S_T"]),
        a["B"], a["T"], a["H"], a["dk"], a["dv"], chunk, _ptr(cu_seqlens), a["n_seqs"], a["io"], float(scale),
        int(snap_every), _ptr(snaps) if n_snap > 0 else None, _ptr(a["workspace"]), a["workspace"].numel(),
        _stream(q.device)))
    return a["o"], a["S_T"], snaps


def gdn_chunk_prefill_snapshots_ex(q, k, v, g, beta, S0=None, *, snap_every, flags=0, chunk=64, cu_seqlens=None,
                                   scale=1.0, o=None, S_T=None, snaps=None, store_state=True, workspace=None):
    """Snapshots with grouped key heads and input transforms; see ``gdn_chunk_prefill_snapshots_ex``.

    Shapes as ``gdn_chunk_prefill_grouped``; returns ``(o, S_T, snaps)`` as ``gdn_chunk_prefill_snapshots``.
    """
    a = _prefill_args(q, k, v, g, beta, S0, chunk, cu_seqlens, o, S_T, store_state, workspace, grouped=True)
    n_snap = max(0, (a["T"] - 1) // (int(snap_every) * chunk)) if snap_every >= 1 else 0
    shape = (a["n"], n_snap, a["H"], a["dv"], a["dk"])
    if snaps is None:
        snaps = torch.zeros(shape, device=q.device, dtype=torch.float32)
    else:
        _dev(snaps, "snaps", torch.float32)
        if tuple(snaps.shape) != shape:
            raise ValueError("snaps must be %s" % (shape,))
    _check(lib().gdn_chunk_prefill_snapshots_ex(
        _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(S0), _ptr(a["o"]), _ptr(a["S_T"]),
        a["B"], a["T"], a["H"], a["HK"], a["dk"], a["dv"], chunk, _ptr(cu_seqlens), a["n_seqs"], a["io"],
        float(scale), int(flags), int(snap_every), _ptr(snaps) if n_snap > 0 else None, _ptr(a["workspace"]),
        a["workspace"].numel(), _stream(q.device)))
    return a["o"], a["S_T"], snaps


def gdn_decode_step(q, k, v, g, beta, S, *, scale=1.0, o=None):
    """One decode step; ``S`` [B,H,dv,dk] fp32 is updated in place.  Returns o [B,H,dv]."""
    return _decode(q, k, v, g, beta, S, scale, o, grouped=False)


def gdn_decode_step_grouped(q, k, v, g, beta, S, *, scale=1.0, o=None):
    """One decode step with grouped key heads: q, k [B,H_k,dk], v [B,H,dv]; ``S`` updated in place.  Returns o."""
    return _decode(q, k, v, g, beta, S, scale, o, grouped=True)


def gdn_decode_step_ex(q, k, v, g, beta, S, *, flags=0, scale=1.0, o=None):
    """One decode step with in-kernel input transforms (``flags`` as ``gdn_chunk_prefill_ex``).  Returns o."""
    return _decode(q, k, v, g, beta, S, scale, o, grouped=True, flags=flags)


def _decode(q, k, v, g, beta, S, scale, o, grouped, flags=None):
    if q.dtype not in _IO:
        raise TypeError("q must be float32 or bfloat16")
    io = _IO[q.dtype]
    for name, t in (("q", q), ("k", k), ("v", v)):
        _dev(t, name, q.dtype)
    _dev(g, "g", torch.float32)
    _dev(beta, "beta", torch.float32)
    _dev(S, "S", torch.float32)
    B, HK, dk = q.shape
    H = v.shape[1] if grouped else HK
    dv = v.shape[-1]
    if k.shape != q.shape or v.shape[:2] != (B, H) or g.shape != (B, H) or beta.shape != g.shape \
            or S.shape != (B, H, dv, dk):
        raise ValueError("inconsistent decode shapes")
    if o is None:
        o = torch.empty_like(v)
    else:
        _dev(o, "o", q.dtype)
    if flags is not None:
        _check(lib().gdn_decode_step_ex(_ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(S), _ptr(o),
                                        B, H, HK, dk, dv, io, float(scale), int(flags), _stream(q.device)))
    elif grouped:
        _check(lib().gdn_decode_step_grouped(_ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(S), _ptr(o),
                                             B, H, HK, dk, dv, io, float(scale), _stream(q.device)))
    else:
        _check(lib().gdn_decode_step(_ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(S), _ptr(o),
                                     B, H, dk, dv, io, float(scale), _stream(q.device)))
    return o


def gdn_attention_prefill(q, k, v, *, scale=None, cu_seqlens=None, o=None):
    """Causal softmax attention; see ``gdn_attention_prefill`` in include/gdn.h.

    q [B,T,H,d] and k, v [B,T,H_kv,d] bf16 CUDA tensors; ``scale`` defaults to
    1/sqrt(d).  Packed sequences: B == 1 and ``cu_seqlens`` an int32 CUDA tensor
    [n+1].  Returns o [B,T,H,d] bf16.
    """
    n_seqs = 0
    if cu_seqlens is not None:
        _dev(cu_seqlens, "cu_seqlens", torch.int32)
        n_seqs = cu_seqlens.numel() - 1
    for name, t in (("q", q), ("k", k), ("v", v)):
        _dev(t, name, torch.bfloat16)
    B, T, H, d = q.shape
    Hkv = k.shape[2]
    if tuple(k.shape) != (B, T, Hkv, d) or v.shape != k.shape:
        raise ValueError("inconsistent shapes q%s k%s v%s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    if o is None:
        o = torch.empty_like(q)
    else:
        _dev(o, "o", torch.bfloat16)
    sc = float(scale) if scale is not None else 1.0 / float(d) ** 0.5
    _check(lib().gdn_attention_prefill(_ptr(q), _ptr(k), _ptr(v), _ptr(o), B, T, H, Hkv, d, _ptr(cu_seqlens), n_seqs,
                                       GDN_BF16, sc, _stream(q.device)))
    return o


# The serving operators are called once or twice a layer and token, where a microsecond counts: one pass over a call's
# tensors checks them and takes their addresses, and what is wrong is only looked for once something is.
_BF16, _F32, _F64, _I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


def _addresses(dev, tensors, names, dtypes):
    """The addresses (None for None) of contiguous tensors of these types on device number ``dev``."""
    out = []
    try:
        for t, dtype in zip(tensors, dtypes):
            if t is None:
                out.append(None)
            elif t.dtype is dtype and t.get_device() == dev and t.is_contiguous():
                out.append(t.data_ptr())
            else:
                break
        else:
            return out
    except AttributeError:   # no tensor
        pass
    name, dtype = names[len(out)], dtypes[len(out)]
    t = _dev(tensors[len(out)], name, dtype)
    raise ValueError("%s is on %s, the call's first tensor on device %d" % (name, t.device, dev))


def _rows(t, name, dtype):
    """(address, elements between neighbouring tokens, device) of t [B,T,heads,d]: a token's rows contiguous, tokens
    equally far apart."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != 4:
        raise ValueError("%s must be [B, T, heads, d], got %s" % (name, tuple(t.shape)))
    B, T, h, d = t.shape
    step = h * d
    if not t.is_contiguous():
        sb, st, sh, sd = t.stride()
        if (sd != 1 and d > 1) or (sh != d and h > 1) or (B > 1 and T > 1 and sb != T * st):
            raise ValueError("%s: a token's rows must be contiguous and the tokens equally far apart" % name)
        step = st if T > 1 else sb if B > 1 else step
    return t.data_ptr(), step, t.get_device()


def _shaped(t, name, shape):
    if t is not None and t.shape != shape:
        raise ValueError("%s must be %s, got %s" % (name, tuple(shape), tuple(t.shape)))


def _on(dev, call, *args):
    """call(*args, the current stream of device ``dev``), with that device current."""
    if dev == torch._C._cuda_getDevice():
        status = call(*args, _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream(dev).cuda_stream)
    else:
        with torch.cuda.device(dev):
            status = call(*args, torch.cuda.current_stream(dev).cuda_stream)
    if status != 0:
        _check(status)


_NORM_NAMES = ("q_out", "k_out", "q_weight", "k_weight", "inv_freq", "positions", "cu_seqlens")


def gdn_qk_norm_rope(q, k, *, q_weight=None, k_weight=None, eps=1e-6, inv_freq=None, interleaved=False, positions=None,
                     cu_seqlens=None, q_out=None, k_out=None):
    """Norms of queries and keys per head and the position rotation; see ``gdn_qk_norm_rope`` in include/gdn.h.

    q [B,T,H,d] and k [B,T,H_kv,d], bf16 or fp32 CUDA tensors, may be parts of a wider projection's rows;
    ``q_weight``, ``k_weight`` [d] fp32; ``inv_freq`` [rot/2] float64; ``positions`` [B,T] int32 (default: a token's
    index in its sequence).  Returns (q_out, k_out), contiguous.
    """
    if not isinstance(q, torch.Tensor) or q.dtype not in _IO:
        raise TypeError("q must be float32 or bfloat16")
    io = q.dtype
    qp, qs, dev = _rows(q, "q", io)
    kp, ks, kdev = _rows(k, "k", io)
    shape = B, T, H, d = q.shape
    Hkv = k.shape[2]
    if k.shape != (B, T, Hkv, d):
        raise ValueError("inconsistent shapes q%s k%s" % (tuple(q.shape), tuple(k.shape)))
    if kdev != dev:
        raise ValueError("q is on %s, k on %s" % (q.device, k.device))
    if q_out is None:
        q_out = torch.empty(shape, device=q.device, dtype=io)
    if k_out is None:
        k_out = torch.empty(k.shape, device=k.device, dtype=io)
    qo, ko, qw, kw, fp, pos, cu = _addresses(dev, (q_out, k_out, q_weight, k_weight, inv_freq, positions, cu_seqlens),
                                             _NORM_NAMES, (io, io, _F32, _F32, _F64, _I32, _I32))
    _shaped(q_out, "q_out", shape)
    _shaped(k_out, "k_out", k.shape)
    _shaped(q_weight, "q_weight", (d,))
    _shaped(k_weight, "k_weight", (d,))
    _shaped(positions, "positions", (B, T))
    _on(dev, lib().gdn_qk_norm_rope, qp, kp, qo, ko, B, T, H, Hkv, d, qs, ks, qw, kw, eps, fp,
        0 if inv_freq is None else 2 * inv_freq.numel(), pos, cu, 0 if cu is None else cu_seqlens.numel() - 1, _IO[io],
        GDN_ROPE_INTERLEAVED if interleaved else 0)
    return q_out, k_out


_CACHE_NAMES = ("k_cache", "v_cache", "block_table", "seq_lens", "cu_seqlens", "k_scale", "v_scale")


def _cache_args(dev, k_cache, v_cache, block_table, seq_lens, cu_seqlens, k_scale, v_scale, B, Hkv, d):
    """Addresses of the cache and its tables, and its sizes; Hkv None: the cache's."""
    ct = _CACHE.get(k_cache.dtype) if isinstance(k_cache, torch.Tensor) else None
    if ct is None:
        raise TypeError("k_cache must be bfloat16 or float8_e4m3fn")
    kind = k_cache.dtype
    at = _addresses(dev, (k_cache, v_cache, block_table, seq_lens, cu_seqlens, k_scale, v_scale), _CACHE_NAMES,
                    (kind, kind, _I32, _I32, _I32, _F32, _F32))
    if None in at[:4]:
        raise TypeError("%s must be a CUDA (HIP) tensor" % _CACHE_NAMES[at.index(None)])
    shape, table = k_cache.shape, block_table.shape
    n_seqs = 0 if cu_seqlens is None else cu_seqlens.numel() - 1
    n = B if cu_seqlens is None else n_seqs
    if len(shape) != 4 or shape[3] != d or (Hkv is not None and shape[1] != Hkv) or v_cache.shape != shape:
        raise ValueError("k_cache and v_cache must be [n_pages, %s, page, %d], got %s and %s" % (
            "H_kv" if Hkv is None else Hkv, d, tuple(shape), tuple(v_cache.shape)))
    if len(table) != 2 or table[0] != n or seq_lens.shape != (n,):
        raise ValueError("block_table must be [%d, max_pages] and seq_lens [%d], got %s and %s" % (
            n, n, tuple(table), tuple(seq_lens.shape)))
    if ct == GDN_E4M3:
        if k_scale is None or v_scale is None:
            raise ValueError("a float8_e4m3fn cache needs k_scale and v_scale")
        _shaped(k_scale, "k_scale", shape[:2])
        _shaped(v_scale, "v_scale", shape[:2])
    elif k_scale is not None or v_scale is not None:
        raise ValueError("k_scale and v_scale belong to a float8_e4m3fn cache")
    return at, shape[1], shape[2], shape[0], table[1], n_seqs, ct


_APPEND_NAMES = ("q_out", "q_weight", "k_weight", "inv_freq")


def gdn_kv_append(k, v, k_cache, v_cache, block_table, seq_lens, *, q=None, q_out=None, k_scale=None, v_scale=None,
                  q_weight=None, k_weight=None, eps=1e-6, inv_freq=None, interleaved=False, cu_seqlens=None):
    """New tokens' keys and values into a paged cache; see ``gdn_kv_append`` in include/gdn.h.

    k, v [B,T,H_kv,d] (and q [B,T,H,d]) bf16, parts of a wider projection's rows or not; caches
    [n_pages,H_kv,page,d] bf16 or float8_e4m3fn, updated in place, with ``k_scale``, ``v_scale`` [n_pages,H_kv] fp32 for
    the latter; ``block_table`` [n,max_pages] and ``seq_lens`` [n] (with the new tokens) int32.  Norm and rotation as
    ``gdn_qk_norm_rope``.  Returns q_out (None without q).
    """
    kp, ks, dev = _rows(k, "k", _BF16)
    vp, vs, vdev = _rows(v, "v", _BF16)
    shape = B, T, Hkv, d = k.shape
    if v.shape != shape:
        raise ValueError("inconsistent shapes k%s v%s" % (tuple(k.shape), tuple(v.shape)))
    qp, qs, qdev, H = None, 0, dev, Hkv
    if q is not None:
        qp, qs, qdev = _rows(q, "q", _BF16)
        H = q.shape[2]
        if q.shape != (B, T, H, d):
            raise ValueError("inconsistent shapes q%s k%s" % (tuple(q.shape), tuple(k.shape)))
        if q_out is None:
            q_out = torch.empty(q.shape, device=q.device, dtype=_BF16)
        elif q_out.shape != q.shape:
            _shaped(q_out, "q_out", q.shape)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if vdev != dev or qdev != dev:
        raise ValueError("q, k and v must be on one device")
    qo, qw, kw, fp = _addresses(dev, (q_out, q_weight, k_weight, inv_freq), _APPEND_NAMES, (_BF16, _F32, _F32, _F64))
    if qw is not None and q_weight.numel() != d:
        _shaped(q_weight, "q_weight", (d,))
    if kw is not None and k_weight.numel() != d:
        _shaped(k_weight, "k_weight", (d,))
    (kc, vc, table, lens, cu, ksc, vsc), _, page, n_pages, max_pages, n_seqs, ct = _cache_args(
        dev, k_cache, v_cache, block_table, seq_lens, cu_seqlens, k_scale, v_scale, B, Hkv, d)
    _on(dev, lib().gdn_kv_append, qp, kp, vp, qo, kc, vc, ksc, vsc, table, lens, B, T, H, Hkv, d, page, n_pages, max_pages,
        qs, ks, vs, qw, kw, eps, fp, 0 if fp is None else 2 * inv_freq.numel(), cu, n_seqs, GDN_BF16, ct,
        GDN_ROPE_INTERLEAVED if interleaved else 0)
    return q_out


def gdn_attention_paged_workspace_bytes(B, T, H, H_kv, d, page, max_pages, n_seqs=0) -> int:
    return int(lib().gdn_attention_paged_workspace_bytes(B, T, H, H_kv, d, page, max_pages, n_seqs))


_ATTENTION_NAMES = ("q", "o", "workspace")


def gdn_attention_paged(q, k_cache, v_cache, block_table, seq_lens, *, k_scale=None, v_scale=None, scale=None,
                        cu_seqlens=None, o=None, workspace=None):
    """Causal attention of new tokens over a paged cache; see ``gdn_attention_paged`` in include/gdn.h.

    q [B,T,H,d] bf16, T new tokens for each of B sequences, or packed (B == 1) with ``cu_seqlens`` int32 [n+1]; the cache
    and its tables as ``gdn_kv_append``, which has put the new tokens there; ``scale`` defaults to 1/sqrt(d).  Returns o.
    """
    _dev(q, "q", _BF16)
    if q.dim() != 4:
        raise ValueError("q must be [B, T, heads, d], got %s" % (tuple(q.shape),))
    shape = B, T, H, d = q.shape
    dev = q.get_device()
    if o is None:
        o = torch.empty(shape, device=q.device, dtype=_BF16)
    (kc, vc, table, lens, cu, ksc, vsc), Hkv, page, n_pages, max_pages, n_seqs, ct = _cache_args(
        dev, k_cache, v_cache, block_table, seq_lens, cu_seqlens, k_scale, v_scale, B, None, d)
    if workspace is None:
        need = lib().gdn_attention_paged_workspace_bytes(B, T, H, Hkv, d, page, max_pages, n_seqs)
        workspace = torch.empty(need, device=q.device, dtype=torch.uint8) if need else None
    qp, op, ws = _addresses(dev, (q, o, workspace), _ATTENTION_NAMES, (_BF16, _BF16, torch.uint8))
    if o.shape != shape:
        _shaped(o, "o", shape)
    size = 0 if ws is None else workspace.numel()
    _on(dev, lib().gdn_attention_paged, qp, kc, vc, ksc, vsc, table, lens, op, B, T, H, Hkv, d, page, n_pages, max_pages, cu,
        n_seqs, GDN_BF16, ct, d ** -0.5 if scale is None else scale, ws if size else None, size)
    return o
