"""Binding of the operators around the mixers: gated linear recurrence.

As in ``binding``: arguments are checked and marshalled here, every step of the operators runs inside ``libhyena.so``, device
memory and streams are PyTorch's, and a failed call raises ``HyenaError``.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import HY_OK, HyenaError, _dtype_code, _on, _stream, lib

GLR_MARK_ROWS = 64  # HYENA_GLR_MARK_ROWS


def declare(L: ctypes.CDLL) -> None:
    """Argument types of this module's entry points."""
    vp, i64, i32, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int
    L.hyena_glr_fwd.argtypes = [vp] * 10 + [i64, i64, i64, i64, i32, ci, vp]
    L.hyena_glr_bwd.argtypes = [vp] * 15 + [i64, i64, i64, i64, i32, ci, vp]
    L.hyena_glr_step.argtypes = [vp] * 6 + [i64, i64, i32, ci, vp]
    for name in ("hyena_glr_fwd", "hyena_glr_bwd", "hyena_glr_step"):
        getattr(L, name).restype = ci
    L.hyena_glr_fwd_workspace_bytes.argtypes = [i64, i64, i64, i32, ci]
    L.hyena_glr_bwd_workspace_bytes.argtypes = [i64, i64, i64, i32, ci, i32]
    for name in ("hyena_glr_fwd_workspace_bytes", "hyena_glr_bwd_workspace_bytes"):
        getattr(L, name).restype = i64


# ---- gated linear recurrence


def _glr_input(name: str, t: torch.Tensor, shape, ref: torch.Tensor) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a tensor on the GPU" % name)
    if t.shape != shape or t.dtype != ref.dtype or t.get_device() != ref.get_device():
        raise ValueError("%s must be %s, of the first tensor's dtype and on its GPU" % (name, list(shape)))
    if shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("%s must have contiguous channels" % name)


def _glr_shapes(first: torch.Tensor, group: int, dims: int):
    """Shapes of an activation and of the log decays."""
    if not isinstance(first, torch.Tensor) or not first.is_cuda:
        raise ValueError("the first activation must be a tensor on the GPU")
    if first.dim() != dims:
        raise ValueError("activations must be %s tensors" % ("[B, L, D]" if dims == 3 else "[B, D]"))
    D = first.shape[-1]
    if group < 1 or D % group != 0:
        raise ValueError("group must divide the width")
    return first.shape, first.shape[:-1] + (D // group,)


def _glr_state(name: str, t, B: int, D: int, ref: torch.Tensor):
    """The pointer of a [B, D] fp32 state, or None."""
    if t is None:
        return None
    if (not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or t.shape != (B, D) or not t.is_contiguous()
            or t.get_device() != ref.get_device()):
        raise ValueError("%s must be a contiguous float32 [B, D] tensor on the same GPU" % name)
    return t.data_ptr()


def _strides(tensors):
    """Distances between batch items and between steps of each tensor; None where all are dense."""
    if all(t.is_contiguous() for t in tensors):
        return None
    return (ctypes.c_int64 * (2 * len(tensors)))(*(d for t in tensors for d in t.stride()[:2]))


def _workspace(need: int, given, ref: torch.Tensor):
    """(pointer, bytes, the tensor that owns them) of a call's workspace."""
    if need < 0:
        raise ValueError("not a valid problem")
    if need == 0:
        return None, 0, None
    if given is None:
        given = torch.empty(need, dtype=torch.uint8, device=ref.device)  # device memory from PyTorch
    elif given.get_device() != ref.get_device() or not given.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the same GPU")
    return given.data_ptr(), given.numel() * given.element_size(), given


def _ptr(t):
    return None if t is None else t.data_ptr()


def _output(t, shape, ref: torch.Tensor, name: str):
    if t is None:
        return torch.empty(shape, dtype=ref.dtype, device=ref.device)
    _glr_input(name, t, shape, ref)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t


def _glr_fwd(q, k, v, g, group, state_in, want_state, want_marks, out, workspace, stream):
    shape, gates = _glr_shapes(q, group, 3)
    code = _dtype_code(q)
    for name, t, s in (("q", q, shape), ("k", k, shape), ("v", v, shape), ("g", g, gates)):
        _glr_input(name, t, s, q)
    B, L, D = shape
    y = _output(out, shape, q, "out")
    state = torch.empty((B, D), dtype=torch.float32, device=q.device) if want_state else None
    marks = torch.empty((B, -(-L // GLR_MARK_ROWS), D), dtype=torch.float32, device=q.device) if want_marks else None
    before = _glr_state("state_in", state_in, B, D, q)
    lb = lib()
    ws, nbytes, keep = _workspace(int(lb.hyena_glr_fwd_workspace_bytes(B, L, D, group, code)), workspace, q)
    with _on(q):
        rc = lb.hyena_glr_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), before, y.data_ptr(), _ptr(state),
                              _ptr(marks), _strides((q, k, v, g)), ws, nbytes, B, L, D, group, code, _stream(q, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_glr_fwd")
    return y, state, marks


def hyena_glr_fwd(q, k, v, g, group: int = 1, out=None, workspace=None, stream=None) -> torch.Tensor:
    """y = q * s with s[t] = exp(g[t]) s[t-1] + k[t] v[t] from a zero state; ``g`` is [B, L, D // group].  Inputs may be views
    whose channels are contiguous; see ``hyena_glr_fwd`` in hyena.h."""
    return _glr_fwd(q, k, v, g, int(group), None, False, False, out, workspace, stream)[0]


def hyena_glr_fwd_carry(q, k, v, g, group: int = 1, state_in=None, want_state: bool = True, want_marks: bool = False, out=None,
                        workspace=None, stream=None):
    """(y, state_out, marks): one stretch of a longer sequence, from the float32 [B, D] state the previous stretch returned
    (None: its start).  ``marks`` is what ``hyena_glr_bwd`` takes; each of the last two is None where it is not wanted."""
    return _glr_fwd(q, k, v, g, int(group), state_in, want_state, want_marks, out, workspace, stream)


def hyena_glr_bwd(dy, q, k, v, g, group: int = 1, marks=None, state_in=None, dstate_out=None, want_dstate: bool = False,
                  workspace=None, stream=None):
    """(dq, dk, dv, dg, dstate_in) of ``hyena_glr_fwd_carry``; ``marks`` as it returned them, or None and ``state_in`` as it was
    given.  dstate_in is None unless ``want_dstate``; see ``hyena_glr_bwd`` in hyena.h."""
    group = int(group)
    shape, gates = _glr_shapes(dy, group, 3)
    code = _dtype_code(dy)
    for name, t, s in (("dy", dy, shape), ("q", q, shape), ("k", k, shape), ("v", v, shape), ("g", g, gates)):
        _glr_input(name, t, s, dy)
    B, L, D = shape
    if marks is not None and (marks.dtype != torch.float32 or marks.shape != (B, -(-L // GLR_MARK_ROWS), D)
                              or not marks.is_contiguous() or marks.get_device() != dy.get_device()):
        raise ValueError("marks must be the tensor that the forward call returned")
    before, behind = _glr_state("state_in", state_in, B, D, dy), _glr_state("dstate_out", dstate_out, B, D, dy)
    dq, dk, dv = (torch.empty(shape, dtype=dy.dtype, device=dy.device) for _ in range(3))
    dg = torch.empty(gates, dtype=dy.dtype, device=dy.device)
    dstate = torch.empty((B, D), dtype=torch.float32, device=dy.device) if want_dstate else None
    lb = lib()
    ws, nbytes, keep = _workspace(int(lb.hyena_glr_bwd_workspace_bytes(B, L, D, group, code, marks is not None)), workspace, dy)
    with _on(dy):
        rc = lb.hyena_glr_bwd(dy.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), _ptr(marks), before, behind,
                              dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dg.data_ptr(), _ptr(dstate),
                              _strides((dy, q, k, v, g)), ws, nbytes, B, L, D, group, code, _stream(dy, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_glr_bwd")
    return dq, dk, dv, dg, dstate


def hyena_glr_step(q, k, v, g, state, group: int = 1, out=None, stream=None) -> torch.Tensor:
    """One token of B sequences: updates the float32 [B, D] ``state`` in place and returns y [B, D]; see ``hyena_glr_step`` in
    hyena.h."""
    group = int(group)
    shape, gates = _glr_shapes(q, group, 2)
    code = _dtype_code(q)
    for name, t, s in (("q", q, shape), ("k", k, shape), ("v", v, shape), ("g", g, gates)):
        _glr_input(name, t, s, q)
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
    B, D = shape
    if state is None:
        raise ValueError("state must be a contiguous float32 [B, D] tensor on the same GPU")
    st = _glr_state("state", state, B, D, q)
    y = _output(out, shape, q, "out")
    with _on(q):
        rc = lib().hyena_glr_step(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), st, y.data_ptr(), B, D, group, code,
                                  _stream(q, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_glr_step")
    return y
