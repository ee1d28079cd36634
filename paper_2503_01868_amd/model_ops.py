"""Binding of the operators around the mixers: gated linear recurrence, cross entropy over a vocabulary,
AdamW.

As in ``binding``: arguments are checked and marshalled here, every step of the operators runs inside ``libhyena.so``, device
memory and streams are PyTorch's, and a failed call raises ``HyenaError``.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import _HERE, HY_OK, HyenaError, _dtype_code, _on, _stream, lib

GLR_MARK_ROWS = 64  # HYENA_GLR_MARK_ROWS


def declare(L: ctypes.CDLL) -> None:
    """Argument types of this module's entry points."""
    vp, i64, i32, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int
    L.hyena_glr_fwd.argtypes = [vp] * 10 + [i64, i64, i64, i64, i32, ci, vp]
    L.hyena_glr_bwd.argtypes = [vp] * 15 + [i64, i64, i64, i64, i32, ci, vp]
    L.hyena_glr_step.argtypes = [vp] * 6 + [i64, i64, i32, ci, vp]
    L.hyena_xent_fwd.argtypes = [vp] * 6 + [i64, i64, i64, i64, ci, vp]
    L.hyena_xent_bwd.argtypes = [vp] * 8 + [i64, i64, i64, i64, ci, vp]
    L.hyena_adamw_table.argtypes = [vp, i64, ci, ci, ci, ci, vp, i64, vp]
    L.hyena_adamw_step.argtypes = [vp, i64, i64, ci, ci, ci, ci] + [ctypes.c_double] * 4 + [i64, vp, vp]
    for name in ("hyena_glr_fwd", "hyena_glr_bwd", "hyena_glr_step", "hyena_xent_fwd", "hyena_xent_bwd", "hyena_adamw_table",
                 "hyena_adamw_step"):
        getattr(L, name).restype = ci
    L.hyena_glr_fwd_workspace_bytes.argtypes = [i64, i64, i64, i32, ci]
    L.hyena_glr_bwd_workspace_bytes.argtypes = [i64, i64, i64, i32, ci, i32]
    L.hyena_xent_fwd_workspace_bytes.argtypes = L.hyena_xent_bwd_workspace_bytes.argtypes = [i64, i64, i64, ci]
    L.hyena_adamw_table_bytes.argtypes = [vp, i64]
    for name in ("hyena_glr_fwd_workspace_bytes", "hyena_glr_bwd_workspace_bytes", "hyena_xent_fwd_workspace_bytes",
                 "hyena_xent_bwd_workspace_bytes", "hyena_adamw_table_bytes"):
        getattr(L, name).restype = i64


def _under(x: torch.Tensor, stream):
    """Context in which memory comes from the pool of the stream that the call runs on."""
    if stream is None:
        return _HERE
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(_stream(x, stream), device=x.device)
    return torch.cuda.stream(stream)


# ---- gated linear recurrence


def _glr_input(name: str, t: torch.Tensor, shape, ref: torch.Tensor) -> None:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a tensor on the GPU" % name)
    if t.shape != shape or t.dtype != ref.dtype or t.get_device() != ref.get_device():
        raise ValueError("%s must be %s, of the first tensor's dtype and on its GPU" % (name, list(shape)))
    if shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("%s must have contiguous channels" % name)


def _glr_inputs(named, ref: torch.Tensor) -> None:
    """_glr_input of every (name, tensor, shape); the flags alone where they are as they mostly are."""
    dtype, gpu = ref.dtype, ref.get_device()
    for name, t, shape in named:
        if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == gpu and t.shape == shape
                and t.is_contiguous()):
            _glr_input(name, t, shape, ref)


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
    _glr_inputs((("q", q, shape), ("k", k, shape), ("v", v, shape), ("g", g, gates)), q)
    B, L, D = shape
    before = _glr_state("state_in", state_in, B, D, q)
    lb = lib()
    with _on(q), _under(q, stream):
        y = _output(out, shape, q, "out")
        state = torch.empty((B, D), dtype=torch.float32, device=q.device) if want_state else None
        marks = torch.empty((B, -(-L // GLR_MARK_ROWS), D), dtype=torch.float32, device=q.device) if want_marks else None
        ws, nbytes, keep = _workspace(int(lb.hyena_glr_fwd_workspace_bytes(B, L, D, group, code)), workspace, q)
        rc = lb.hyena_glr_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), before, y.data_ptr(), _ptr(state),
                              _ptr(marks), _strides((q, k, v, g)), ws, nbytes, B, L, D, group, code, _stream(q, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_glr_fwd")
    return y, state, marks


def hyena_glr_fwd(q, k, v, g, group: int = 1, out=None, workspace=None, stream=None) -> torch.Tensor:
    """y = q * s with s[t] = exp(g[t]) s[t-1] + k[t] v[t] from a zero state; ``g`` is [B, L, D // group].  A decay of
    zero forgets everything before its step, NaN included.  Inputs may be views whose channels are contiguous; see
    ``hyena_glr_fwd`` in hyena.h."""
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
    _glr_inputs((("dy", dy, shape), ("q", q, shape), ("k", k, shape), ("v", v, shape), ("g", g, gates)), dy)
    B, L, D = shape
    if marks is not None and (marks.dtype != torch.float32 or marks.shape != (B, -(-L // GLR_MARK_ROWS), D)
                              or not marks.is_contiguous() or marks.get_device() != dy.get_device()):
        raise ValueError("marks must be the tensor that the forward call returned")
    before, behind = _glr_state("state_in", state_in, B, D, dy), _glr_state("dstate_out", dstate_out, B, D, dy)
    lb = lib()
    with _on(dy), _under(dy, stream):
        dq, dk, dv = (torch.empty(shape, dtype=dy.dtype, device=dy.device) for _ in range(3))
        dg = torch.empty(gates, dtype=dy.dtype, device=dy.device)
        dstate = torch.empty((B, D), dtype=torch.float32, device=dy.device) if want_dstate else None
        need = int(lb.hyena_glr_bwd_workspace_bytes(B, L, D, group, code, marks is not None))
        ws, nbytes, keep = _workspace(need, workspace, dy)
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
    _glr_inputs((("q", q, shape), ("k", k, shape), ("v", v, shape), ("g", g, gates)), q)
    for name, t in (("q", q), ("k", k), ("v", v), ("g", g)):
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
    B, D = shape
    if state is None:
        raise ValueError("state must be a contiguous float32 [B, D] tensor on the same GPU")
    st = _glr_state("state", state, B, D, q)
    with _on(q), _under(q, stream):
        y = torch.empty_like(q) if out is None else _output(out, shape, q, "out")
        rc = lib().hyena_glr_step(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), st, y.data_ptr(), B, D, group, code,
                                  _stream(q, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_glr_step")
    return y


# ---- cross entropy over a vocabulary


def _xent_inputs(x, w, target):
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dim() != 2 or not x.is_contiguous():
        raise ValueError("x must be a contiguous [N, D] tensor on the GPU")
    if (not isinstance(w, torch.Tensor) or w.dim() != 2 or not w.is_contiguous() or w.shape[1] != x.shape[1]
            or w.dtype != x.dtype or w.get_device() != x.get_device()):
        raise ValueError("w must be a contiguous [V, D] tensor of x's dtype on its GPU")
    if (not isinstance(target, torch.Tensor) or target.dtype != torch.int64 or target.shape != x.shape[:1]
            or not target.is_contiguous() or target.get_device() != x.get_device()):
        raise ValueError("target must be a contiguous int64 [N] tensor on x's GPU")
    return x.shape[0], w.shape[0], x.shape[1], _dtype_code(x)


def _xent_column(name, t, N, x):
    if (not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or t.shape != (N,) or not t.is_contiguous()
            or t.get_device() != x.get_device()):
        raise ValueError("%s must be a contiguous float32 [N] tensor on x's GPU" % name)


def _at_16_bytes(t):
    """A column as the library takes it: one that begins between (tokens[1:], say) is copied."""
    return t if t.data_ptr() % 16 == 0 else t.clone()


def hyena_xent_fwd(x, w, target, workspace=None, stream=None):
    """(loss, lse), float32 [N]: softmax cross entropy of the rows of x w^T with ``target`` (int64; a row whose target is no row
    of w has loss 0).  The logits are not kept; see ``hyena_xent_fwd`` in hyena.h."""
    N, V, D, code = _xent_inputs(x, w, target)
    lb = lib()
    with _on(x), _under(x, stream):
        loss, lse = (torch.empty(N, dtype=torch.float32, device=x.device) for _ in range(2))
        target = _at_16_bytes(target)
        ws, nbytes, keep = _workspace(int(lb.hyena_xent_fwd_workspace_bytes(N, V, D, code)), workspace, x)
        rc = lb.hyena_xent_fwd(x.data_ptr(), w.data_ptr(), target.data_ptr(), loss.data_ptr(), lse.data_ptr(), ws, nbytes, N, V, D,
                               code, _stream(x, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_xent_fwd")
    return loss, lse


def hyena_xent_bwd(dloss, x, w, target, lse, workspace=None, stream=None):
    """(dx, dw) of ``hyena_xent_fwd``, given the gradient of every row's loss (1 / N for a mean) and the ``lse`` it returned; see
    ``hyena_xent_bwd`` in hyena.h."""
    N, V, D, code = _xent_inputs(x, w, target)
    _xent_column("dloss", dloss, N, x)
    _xent_column("lse", lse, N, x)
    lb = lib()
    with _on(x), _under(x, stream):
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        dloss, target, lse = _at_16_bytes(dloss), _at_16_bytes(target), _at_16_bytes(lse)
        ws, nbytes, keep = _workspace(int(lb.hyena_xent_bwd_workspace_bytes(N, V, D, code)), workspace, x)
        rc = lb.hyena_xent_bwd(dloss.data_ptr(), x.data_ptr(), w.data_ptr(), target.data_ptr(), lse.data_ptr(), dx.data_ptr(),
                               dw.data_ptr(), ws, nbytes, N, V, D, code, _stream(x, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_xent_bwd")
    return dx, dw


# ---- AdamW

ADAMW_BLOCK = 256  # HYENA_ADAMW_BLOCK


class _AdamwTensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "exp_avg", "exp_avg_sq", "avg_scale", "sq_scale", "master")] + [
        ("count", ctypes.c_int64), ("weight_decay", ctypes.c_float)]


def adamw_state(params, bits: int = 32, masters: bool = False) -> dict:
    """The states before the first step, as keyword arguments of ``plan_adamw``: float32 moments, or with ``bits`` 8 the first
    moment and the root of the second as float8_e4m3fn tensors with a float32 scale per 256 elements; with ``masters``, float32
    copies of the parameters."""
    if bits not in (8, 32):
        raise ValueError("bits must be 8 or 32")
    kind = torch.float32 if bits == 32 else torch.float8_e4m3fn

    def zeros(dtype, per=1):
        return [torch.zeros(-(-p.numel() // per) if per > 1 else p.shape, dtype=torch.uint8 if dtype.itemsize == 1 else dtype,
                            device=p.device).view(dtype) for p in params]

    state = dict(exp_avg=zeros(kind), exp_avg_sq=zeros(kind))
    if bits == 8:
        state.update(avg_scales=zeros(torch.float32, ADAMW_BLOCK), sq_scales=zeros(torch.float32, ADAMW_BLOCK))
    if masters:
        state["masters"] = [p.detach().float() for p in params]
    return state


def _adamw_list(name, ts, params, dtypes, per=1):
    """The tensors of one kind: one dtype, contiguous, on the parameters' GPU, an element for every ``per`` of a parameter."""
    ts = list(ts)
    if len(ts) != len(params):
        raise ValueError("%s must be one tensor for each parameter" % name)
    for t, p in zip(ts, params):
        if (not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype not in dtypes or t.dtype != ts[0].dtype
                or not t.is_contiguous() or t.get_device() != params[0].get_device() or t.numel() != -(-p.numel() // per)):
            raise ValueError("%s must be contiguous tensors of one dtype (%s) with %s on the parameters' GPU" % (
                name, " or ".join(str(d) for d in dtypes), "a parameter's elements" if per == 1 else "an element per block"))
    return ts


class AdamwPlan:
    """The tensors of ``hyena_adamw_step``, laid out once in a table on the GPU: calling it takes a step.  The tensors are kept
    alive, and must stay where they are (gradients too: zero them in place)."""

    def __init__(self, params, grads, exp_avg, exp_avg_sq, masters=None, avg_scales=None, sq_scales=None, weight_decay=0.0):
        params = list(params)
        plain = (torch.float32, torch.bfloat16)
        params = _adamw_list("params", params, params, plain)
        grads = _adamw_list("grads", grads, params, plain)
        exp_avg = _adamw_list("exp_avg", exp_avg, params, (torch.float32, torch.float8_e4m3fn))
        exp_avg_sq = _adamw_list("exp_avg_sq", exp_avg_sq, params, (exp_avg[0].dtype,) if params else plain)
        narrow = bool(params) and exp_avg[0].dtype == torch.float8_e4m3fn
        if narrow != (avg_scales is not None) or narrow != (sq_scales is not None):
            raise ValueError("8-bit states come with avg_scales and sq_scales, others without")
        n = len(params)
        none = [None] * n
        avg_scales = _adamw_list("avg_scales", avg_scales, params, (torch.float32,), ADAMW_BLOCK) if narrow else none
        sq_scales = _adamw_list("sq_scales", sq_scales, params, (torch.float32,), ADAMW_BLOCK) if narrow else none
        own = none if masters is None else _adamw_list("masters", masters, params, (torch.float32,))
        decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(x) for x in weight_decay]
        if len(decay) != n:
            raise ValueError("weight_decay must be a number or one for each parameter")
        self._keep = (params, grads, exp_avg, exp_avg_sq, avg_scales, sq_scales, own)
        self._kinds = (_dtype_code(params[0]), _dtype_code(grads[0]), 8 if narrow else 32, int(masters is not None)) if n else (
            0, 0, 32, 0)
        rows = (_AdamwTensor * n)(*(_AdamwTensor(*(_ptr(t) for t in ts), ts[0].numel(), wd)
                                    for ts, wd in zip(zip(*self._keep), decay)))
        lb = lib()
        need = int(lb.hyena_adamw_table_bytes(rows, n))
        if need < 0:
            raise ValueError("not a valid problem")
        table, chunks = torch.empty(need, dtype=torch.uint8), ctypes.c_int64()
        rc = lb.hyena_adamw_table(rows, n, *self._kinds, table.data_ptr() if need else None, need, ctypes.byref(chunks))
        if rc != HY_OK:
            raise HyenaError(rc, "hyena_adamw_table")
        self._n, self._chunks = n, chunks.value
        if n:
            with _on(params[0]):
                table = table.to(params[0].device)
                self._home = _stream(params[0], None)  # the stream from whose pool the table is
        self._table = table
        self._fn = lb.hyena_adamw_step

    def __call__(self, lr: float, step: int, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8, grad_scale=None,
                 stream=None) -> None:
        """The ``step``-th step, counted from 1.  ``grad_scale``: a float32 number on the GPU that multiplies the gradients (what
        clipping found, or the inverse of a loss scale)."""
        if not self._n:
            return
        first = self._keep[0][0]
        if grad_scale is not None and (not isinstance(grad_scale, torch.Tensor) or grad_scale.dtype != torch.float32
                                       or grad_scale.numel() != 1 or grad_scale.get_device() != first.get_device()):
            raise ValueError("grad_scale must be one float32 number on the parameters' GPU")
        with _on(first):
            on = _stream(first, stream)
            if on != self._home:  # the table must outlive a step on another stream, also where the plan does not
                self._table.record_stream(torch.cuda.ExternalStream(on, device=first.device))
            rc = self._fn(self._table.data_ptr(), self._n, self._chunks, *self._kinds, lr, beta1, beta2, eps, step,
                          _ptr(grad_scale), on)
        if rc != HY_OK:
            raise HyenaError(rc, "hyena_adamw_step")


def plan_adamw(params, grads, exp_avg, exp_avg_sq, masters=None, avg_scales=None, sq_scales=None, weight_decay=0.0) -> AdamwPlan:
    """Lay out the tensors of an AdamW step for repeated issue: parameters and gradients in float32 or bfloat16, states and
    masters as ``adamw_state`` makes them, ``weight_decay`` one number or one per tensor; see ``hyena_adamw_step`` in hyena.h."""
    return AdamwPlan(params, grads, exp_avg, exp_avg_sq, masters, avg_scales, sq_scales, weight_decay)


def hyena_adamw_step(params, grads, exp_avg, exp_avg_sq, lr: float, step: int, masters=None, avg_scales=None, sq_scales=None,
                     weight_decay=0.0, beta1: float = 0.9, beta2: float = 0.95, eps: float = 1e-8, grad_scale=None,
                     stream=None) -> None:
    """One AdamW step, the table laid out for this call alone (gradients that are new tensors every time)."""
    params = list(params)
    with _under(params[0], stream) if params else _HERE:
        plan_adamw(params, grads, exp_avg, exp_avg_sq, masters, avg_scales, sq_scales, weight_decay)(
            lr, step, beta1, beta2, eps, grad_scale, stream)
