"""Binding of what a recurrent block and a decoder have beside the mixers: linear attention with a decay for each head, the
root-mean-square norm with the residual's addition, and the choice of the next token.

As in ``binding``: arguments are checked and marshalled here, every step of the operators runs inside ``libhyena.so``, device
memory and streams are PyTorch's, and a failed call raises ``HyenaError``.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding
from .binding import HY_OK, HyenaError, _dtype_code, _on, _stream, lib
from .model_ops import _ptr, _under, _workspace


def declare(L: ctypes.CDLL) -> None:
    """Argument types of this module's entry points."""
    vp, i64, i32, f64 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_double
    sizes = [i64, i64, i64, i32, i64, i64]  # B, L, H, group, dk, dv
    L.hyena_la_fwd.argtypes = [vp] * 10 + [i64] + sizes + [f64, i32, vp]
    L.hyena_la_bwd.argtypes = [vp] * 15 + [i64] + sizes + [f64, i32, vp]
    L.hyena_la_step.argtypes = [vp] * 6 + [i64, i64, i32, i64, i64, f64, i32, vp]
    L.hyena_rmsnorm_fwd.argtypes = [vp] * 7 + [i64] * 4 + [f64, i32, vp]
    L.hyena_rmsnorm_bwd.argtypes = [vp] * 8 + [i64] * 3 + [i32, vp]
    L.hyena_sample.argtypes = [vp, vp, vp, f64, vp, i32, vp, f64, vp, f64, vp, vp, i64, i64, i64, i32, vp]
    for name in ("hyena_la_fwd", "hyena_la_bwd", "hyena_la_step", "hyena_rmsnorm_fwd", "hyena_rmsnorm_bwd", "hyena_sample"):
        getattr(L, name).restype = ctypes.c_int
    L.hyena_la_marks_bytes.argtypes = L.hyena_la_fwd_workspace_bytes.argtypes = sizes + [i32]
    L.hyena_la_bwd_workspace_bytes.argtypes = sizes + [i32, i32]
    L.hyena_rmsnorm_bwd_workspace_bytes.argtypes = [i64, i64, i32]
    for name in ("hyena_la_marks_bytes", "hyena_la_fwd_workspace_bytes", "hyena_la_bwd_workspace_bytes",
                 "hyena_rmsnorm_bwd_workspace_bytes"):
        getattr(L, name).restype = i64


def _like(name: str, t, shape, ref: torch.Tensor, dtype=None, dense: bool = True) -> None:
    """A tensor of this shape on the reference's GPU, of its dtype or the one given."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError("%s must be a tensor on the GPU" % name)
    if t.shape != shape or t.dtype != (dtype or ref.dtype) or t.get_device() != ref.get_device():
        raise ValueError("%s must be %s of %s on the first tensor's GPU" % (name, list(shape), dtype or ref.dtype))
    if dense and not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _out(name: str, t, shape, ref: torch.Tensor):
    if t is None:
        return torch.empty(shape, dtype=ref.dtype, device=ref.device)
    _like(name, t, shape, ref)
    return t


# ---- linear attention with a decay for each head


def _la_sizes(q, k, v, g, dims: int):
    """(leading sizes, H, group, dk, dv, dtype code) of the inputs, whose channels are contiguous."""
    for name, t in (("q", q), ("k", k), ("v", v), ("g", g)):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise ValueError("%s must be a tensor on the GPU" % name)
    lead = "[B, L, " if dims == 4 else "[B, "
    if q.dim() != dims or v.dim() != dims or g.dim() != dims - 1:
        raise ValueError("q and k must be %sheads, dk], v %sH, dv] and g %sH] tensors" % (lead, lead, lead))
    H, dv = v.shape[-2:]
    heads, dk = q.shape[-2:]
    if dk < 1 or dv < 1 or (heads == 0) != (H == 0) or (heads and H % heads != 0):
        raise ValueError("the heads of q and k must divide those of v, each at least one number wide")
    at = v.shape[:-2]
    _like("q", q, at + (heads, dk), v, dense=False)
    _like("k", k, at + (heads, dk), v, dense=False)
    _like("g", g, at + (H,), v, dense=False)
    for name, t in (("q", q), ("k", k), ("v", v), ("g", g)):
        if t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel():
            raise ValueError("%s must have contiguous channels" % name)
    return at, H, H // heads if heads else 1, dk, dv, _dtype_code(v)


def _la_state(name: str, t, B, H, dk, dv, ref):
    """The pointer of a [B, H, dk, dv] fp32 state, or None."""
    if t is None:
        return None
    _like(name, t, (B, H, dk, dv), ref, torch.float32)
    return t.data_ptr()


def _la_strides(tensors, g):
    """Distances between batch items, steps and heads of each tensor, and of g's batch items and steps; None where all are dense."""
    if g.is_contiguous() and all(t.is_contiguous() for t in tensors):
        return None
    distances = [d for t in tensors for d in t.stride()[:3]] + list(g.stride()[:2])
    return (ctypes.c_int64 * len(distances))(*distances)


def _la_fwd(q, k, v, g, scale, state_in, want_state, want_marks, out, workspace, stream):
    (B, L), H, group, dk, dv, code = _la_sizes(q, k, v, g, 4)
    before = _la_state("state_in", state_in, B, H, dk, dv, v)
    lb = lib()
    with _on(v), _under(v, stream):
        y = _out("out", out, v.shape, v)
        state = torch.empty((B, H, dk, dv), dtype=torch.float32, device=v.device) if want_state else None
        marks = None
        if want_marks:
            need = int(lb.hyena_la_marks_bytes(B, L, H, group, dk, dv, code))
            if need < 0:
                raise HyenaError(5, "hyena_la_fwd")
            marks = torch.empty(need, dtype=torch.uint8, device=v.device)
        ws, nbytes, keep = _la_workspace(int(lb.hyena_la_fwd_workspace_bytes(B, L, H, group, dk, dv, code)), workspace, v, "hyena_la_fwd")
        rc = lb.hyena_la_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), before, y.data_ptr(), _ptr(state), _ptr(marks),
                             _la_strides((q, k, v), g), ws, nbytes, B, L, H, group, dk, dv, float(scale), code, _stream(v, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_la_fwd")
    return y, state, marks


def _la_workspace(need: int, given, ref, call: str):
    if need < 0:
        raise HyenaError(5, call)  # (the shapes are consistent: sizes that are not served)
    return _workspace(need, given, ref)


def hyena_la_fwd(q, k, v, g, scale: float = 1.0, out=None, workspace=None, stream=None) -> torch.Tensor:
    """y = scale q S with S[t] = exp(g[t]) S[t-1] + k[t]^T v[t] for every head, from a zero state: linear attention whose memory
    decays.  ``v`` is [B, L, H, dv] and ``g``, log decays, [B, L, H]; ``q`` and ``k`` are [B, L, H // group, dk], a head of theirs
    for ``group`` heads of v.  A decay of zero forgets everything before its step, NaN included.  Inputs may be views whose channels
    are contiguous; see ``hyena_la_fwd`` in hyena.h."""
    return _la_fwd(q, k, v, g, scale, None, False, False, out, workspace, stream)[0]


def hyena_la_fwd_carry(q, k, v, g, scale: float = 1.0, state_in=None, want_state: bool = True, want_marks: bool = False, out=None,
                       workspace=None, stream=None):
    """(y, state_out, marks): one stretch of a longer sequence, from the float32 [B, H, dk, dv] state the previous stretch returned
    (None: its start).  ``marks``, bytes that ``hyena_la_bwd`` takes, hold the states inside the stretch; each of the last two is
    None where it is not wanted."""
    return _la_fwd(q, k, v, g, scale, state_in, want_state, want_marks, out, workspace, stream)


def hyena_la_bwd(dy, q, k, v, g, scale: float = 1.0, marks=None, state_in=None, dstate_out=None, want_dstate: bool = False,
                 workspace=None, stream=None):
    """(dq, dk, dv, dg, dstate_in) of ``hyena_la_fwd_carry``; ``marks`` as it returned them, or None and ``state_in`` as it was
    given.  dstate_in is None unless ``want_dstate``; see ``hyena_la_bwd`` in hyena.h."""
    (B, L), H, group, d_k, d_v, code = _la_sizes(q, k, v, g, 4)
    _like("dy", dy, v.shape, v, dense=False)
    if d_v > 1 and dy.stride(-1) != 1 and dy.numel():
        raise ValueError("dy must have contiguous channels")
    before, behind = _la_state("state_in", state_in, B, H, d_k, d_v, v), _la_state("dstate_out", dstate_out, B, H, d_k, d_v, v)
    lb = lib()
    if marks is not None and (not isinstance(marks, torch.Tensor) or marks.dtype != torch.uint8 or not marks.is_contiguous()
                              or marks.get_device() != v.get_device()
                              or marks.numel() != int(lb.hyena_la_marks_bytes(B, L, H, group, d_k, d_v, code))):
        raise ValueError("marks must be the tensor that the forward call returned")
    with _on(v), _under(v, stream):
        dq, dk = (torch.empty(q.shape, dtype=v.dtype, device=v.device) for _ in range(2))
        dv = torch.empty(v.shape, dtype=v.dtype, device=v.device)
        dg = torch.empty(g.shape, dtype=v.dtype, device=v.device)
        dstate = torch.empty((B, H, d_k, d_v), dtype=torch.float32, device=v.device) if want_dstate else None
        need = int(lb.hyena_la_bwd_workspace_bytes(B, L, H, group, d_k, d_v, code, marks is not None))
        ws, nbytes, keep = _la_workspace(need, workspace, v, "hyena_la_bwd")
        rc = lb.hyena_la_bwd(dy.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), _ptr(marks), before, behind,
                             dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), dg.data_ptr(), _ptr(dstate), _la_strides((dy, q, k, v), g),
                             ws, nbytes, B, L, H, group, d_k, d_v, float(scale), code, _stream(v, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_la_bwd")
    return dq, dk, dv, dg, dstate


def hyena_la_step(q, k, v, g, state, scale: float = 1.0, out=None, stream=None) -> torch.Tensor:
    """One token of B sequences: updates the float32 [B, H, dk, dv] ``state`` in place and returns y [B, H, dv], from ``q`` and
    ``k`` [B, H // group, dk], ``v`` [B, H, dv] and ``g`` [B, H]; see ``hyena_la_step`` in hyena.h."""
    if out is None and stream is None:
        y = binding._fast.la_step(q, k, v, g, state, scale)
        if y is not None:
            return y
    (B,), H, group, dk, dv, code = _la_sizes(q, k, v, g, 3)
    for name, t in (("q", q), ("k", k), ("v", v), ("g", g)):
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
    if state is None:
        raise ValueError("state must be a contiguous float32 [B, H, dk, dv] tensor on the same GPU")
    st = _la_state("state", state, B, H, dk, dv, v)
    with _on(v), _under(v, stream):
        y = _out("out", out, v.shape, v)
        rc = lib().hyena_la_step(q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), st, y.data_ptr(), B, H, group, dk, dv,
                                 float(scale), code, _stream(v, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_la_step")
    return y


# ---- root-mean-square norm


def _rows(name: str, t, ref=None):
    """[rows, D] sizes and the distance of rows of a [..., D] tensor whose leading sizes can be walked as one."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() < 1:
        raise ValueError("%s must be a [..., D] tensor on the GPU" % name)
    if ref is not None and (t.shape != ref.shape or t.dtype != ref.dtype or t.get_device() != ref.get_device()):
        raise ValueError("%s must have the first tensor's shape and dtype, on its GPU" % name)
    D = t.shape[-1]
    N = t.numel() // D if D else 0
    if N <= 1 or t.is_contiguous():
        if D > 1 and N > 0 and t.stride(-1) != 1:
            raise ValueError("%s must have contiguous channels" % name)
        return N, D, D
    if t.stride(-1) != 1 and D > 1:
        raise ValueError("%s must have contiguous channels" % name)
    step = None
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if step is None:
            first, step = stride, stride * size
        elif stride != step:
            raise ValueError("%s must have rows the same distance apart" % name)
        else:
            step *= size
    return N, D, first


def _weights(w, x):
    if w is not None:
        _like("w", w, x.shape[-1:], x)


def _norm_fwd(x, w, residual, eps, total, want_rstd, out, eight, stream, call):
    N, D, x_step = _rows("x", x)
    if D < 1:
        raise ValueError("x must have at least one channel")
    _weights(w, x)
    r_step = _rows("residual", residual, x)[2] if residual is not None else 0
    code = _dtype_code(x)
    if total is not None:
        if residual is None:
            raise ValueError("total is the sum with a residual")
        _like("total", total, x.shape, x)
    with _on(x), _under(x, stream):
        if eight:
            y = torch.empty(x.shape, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn)
            scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        else:
            y, scale = _out("out", out, x.shape, x), None
        if residual is not None and total is None:
            total = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if want_rstd else None
        rc = lib().hyena_rmsnorm_fwd(x.data_ptr(), _ptr(residual), _ptr(w), y.data_ptr(), _ptr(scale), _ptr(total), _ptr(rstd), N, D,
                                     x_step, r_step, float(eps), code, _stream(x, stream))
    if rc != HY_OK:
        raise HyenaError(rc, call)
    return y, scale, x if residual is None else total, rstd


def hyena_rmsnorm_fwd(x, w=None, residual=None, eps: float = 1e-6, total=None, want_rstd: bool = False, out=None, stream=None):
    """(y, total, rstd): total = x + residual (x itself without a residual), y = total / sqrt(mean(total^2) + eps) * w over the
    last dimension; ``w`` [D] or None.  ``total``: where the sum goes, the residual itself to add in place.  rstd, float32, is None
    unless ``want_rstd``; ``hyena_rmsnorm_bwd`` takes it and the sum.  x and the residual may be views whose rows are the same
    distance apart; see ``hyena_rmsnorm_fwd`` in hyena.h."""
    if total is None and out is None and stream is None:
        made = binding._fast.norm_fwd(x, w, residual, eps, want_rstd, False)
        if made is not None:
            return made
    y, _, total, rstd = _norm_fwd(x, w, residual, eps, total, want_rstd, out, False, stream, "hyena_rmsnorm_fwd")
    return y, total, rstd


def hyena_rmsnorm_fwd_8bit(x, w=None, residual=None, eps: float = 1e-6, total=None, want_rstd: bool = False, stream=None):
    """(y, scale, total, rstd): ``hyena_rmsnorm_fwd`` with y as float8_e4m3fn numbers and a float32 scale for every row (value =
    number * scale, the row's largest at 448)."""
    if total is None and stream is None:
        made = binding._fast.norm_fwd(x, w, residual, eps, want_rstd, True)
        if made is not None:
            return made
    return _norm_fwd(x, w, residual, eps, total, want_rstd, None, True, stream, "hyena_rmsnorm_fwd")


def hyena_rmsnorm_bwd(dy, total, rstd, w=None, dtotal=None, want_dw: bool = True, dx=None, workspace=None, stream=None):
    """(dx, dw) of ``hyena_rmsnorm_fwd`` (of its 8-bit form too), given what it returned: dx is the gradient of x and of the
    residual alike, with ``dtotal``, what comes back along the residual, added.  ``dx``: where it goes, ``dtotal`` or ``dy``
    themselves to write in place.  dw is None without weights; see ``hyena_rmsnorm_bwd`` in hyena.h."""
    if dx is None and workspace is None and stream is None:
        made = binding._fast.norm_bwd(dy, total, rstd, w, dtotal, want_dw)
        if made is not None:
            return made
    N, D, _ = _rows("dy", dy)
    if D < 1:
        raise ValueError("dy must have at least one channel")
    _like("dy", dy, dy.shape, dy)
    _like("total", total, dy.shape, dy)
    _like("rstd", rstd, dy.shape[:-1], dy, torch.float32)
    _weights(w, dy)
    if dtotal is not None:
        _like("dtotal", dtotal, dy.shape, dy)
    code = _dtype_code(dy)
    lb = lib()
    with _on(dy), _under(dy, stream):
        dx = _out("dx", dx, dy.shape, dy)
        dw = torch.empty_like(w) if w is not None and want_dw else None
        ws, nbytes, keep = _workspace(int(lb.hyena_rmsnorm_bwd_workspace_bytes(N, D, code)) if dw is not None else 0, workspace, dy)
        rc = lb.hyena_rmsnorm_bwd(dy.data_ptr(), total.data_ptr(), rstd.data_ptr(), _ptr(w), _ptr(dtotal), dx.data_ptr(), _ptr(dw), ws,
                                  nbytes, N, D, code, _stream(dy, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_rmsnorm_bwd")
    return dx, dw


# ---- the next token


def _setting(name: str, x, N: int, ref, dtype, otherwise):
    """(pointer, the one value) of a setting that is a number, a tensor with one for every row, or None."""
    if isinstance(x, torch.Tensor):
        _like(name, x, (N,), ref, dtype)
        return x.data_ptr(), otherwise
    return None, otherwise if x is None else type(otherwise)(x)


def hyena_sample(logits, u, temperature=1.0, top_k=None, top_p=None, min_p=None, want_prob: bool = True, stream=None):
    """(token, prob): the next token of every row of ``logits`` [N, V], drawn by the random numbers ``u``, float32 [N] in [0, 1).
    Of the softmax of logits / temperature, the ``top_k`` likeliest words are kept, of them the fewest that have ``top_p`` of the
    weight, of them those with at least ``min_p`` times the likeliest's; the token, int64, is where the running sum of what is kept
    passes u, and prob, float32, the probability it was drawn with (None unless ``want_prob``).  A temperature of 0 takes the largest logit.  Each setting
    is a number, a tensor with one for every row (float32; top_k int32), or None; see ``hyena_sample`` in hyena.h."""
    if want_prob and stream is None:
        made = binding._fast.sample(logits, u, temperature, top_k, top_p, min_p)
        if made is not None:
            return made
    if not isinstance(logits, torch.Tensor) or not logits.is_cuda or logits.dim() != 2 or logits.shape[1] < 1:
        raise ValueError("logits must be a [N, V] tensor on the GPU")
    N, V = logits.shape
    if V > 1 and logits.stride(1) != 1 and N:
        raise ValueError("logits must have contiguous words")
    code = _dtype_code(logits)
    _like("u", u, (N,), logits, torch.float32)
    t = _setting("temperature", temperature, N, logits, torch.float32, 1.0)
    k = _setting("top_k", top_k, N, logits, torch.int32, 0)
    p = _setting("top_p", top_p, N, logits, torch.float32, 1.0)
    m = _setting("min_p", min_p, N, logits, torch.float32, 0.0)
    k = k[0], max(-1, min(k[1], 2 ** 31 - 1))
    with _on(logits), _under(logits, stream):
        token = torch.empty(N, dtype=torch.int64, device=logits.device)
        prob = torch.empty(N, dtype=torch.float32, device=logits.device) if want_prob else None
        rc = lib().hyena_sample(logits.data_ptr(), u.data_ptr(), *t, *k, *p, *m, token.data_ptr(), _ptr(prob), N, V,
                                logits.stride(0) if N > 1 else 0, code, _stream(logits, stream))
    if rc != HY_OK:
        raise HyenaError(rc, "hyena_sample")
    return token, prob
