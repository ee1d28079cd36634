"""Linear attention, the RMS norm and the choice of tokens in 64 bits, written out step by step (numpy)."""
import math

import numpy as np

FORGETS = -87.3


def _heads(x, group):
    return np.repeat(x, group, axis=2)


def _decay(g):
    return np.where(g < FORGETS, 0.0, np.exp(np.minimum(g, 700.0)))


def _kept(a, S):
    """a S, where a decay of zero leaves nothing, whatever S holds."""
    return np.where(a[..., None, None] == 0, 0.0, a[..., None, None] * np.where(a[..., None, None] == 0, 0.0, S))


def la(q, k, v, g, group=1, scale=1.0, state=None):
    """(y, state after the last step)."""
    B, L, H, dv = v.shape
    q, k, a = _heads(q, group), _heads(k, group), _decay(g)
    S = np.zeros((B, H, q.shape[3], dv)) if state is None else state.astype(np.float64).copy()
    y = np.zeros((B, L, H, dv))
    for t in range(L):
        S = _kept(a[:, t], S) + k[:, t, :, :, None] * v[:, t, :, None, :]
        y[:, t] = scale * np.einsum("bhd,bhdc->bhc", q[:, t], S)
    return y, S


def la_grads(dy, q, k, v, g, group=1, scale=1.0, state=None, dstate=None):
    """(dq, dk, dv, dg, dstate_in)."""
    B, L, H, dv_ = v.shape
    hk, dk_ = q.shape[2:]
    q, k, a = _heads(q, group), _heads(k, group), _decay(g)
    S = np.zeros((B, H, dk_, dv_)) if state is None else state.astype(np.float64).copy()
    every = [S]
    for t in range(L):
        S = _kept(a[:, t], S) + k[:, t, :, :, None] * v[:, t, :, None, :]
        every.append(S)
    M = np.zeros((B, H, dk_, dv_)) if dstate is None else dstate.astype(np.float64).copy()
    dq, dk, dv, dg = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape), np.zeros(g.shape)
    for t in range(L - 1, -1, -1):
        M = M + scale * q[:, t, :, :, None] * dy[:, t, :, None, :]
        dq[:, t] = scale * np.einsum("bhc,bhdc->bhd", dy[:, t], every[t + 1])
        dk[:, t] = np.einsum("bhc,bhdc->bhd", v[:, t], M)
        dv[:, t] = np.einsum("bhd,bhdc->bhc", k[:, t], M)
        dg[:, t] = np.einsum("bhdc,bhdc->bh", _kept(a[:, t], every[t]), np.where(a[:, t, :, None, None] == 0, 0.0, M))
        M = _kept(a[:, t], M)
    share = lambda x: x.reshape(B, L, hk, group, dk_).sum(3)  # noqa: E731
    return share(dq), share(dk), dv, dg, M


def rmsnorm(x, w=None, residual=None, eps=1e-6):
    """(y, h, rstd); the sum is not rounded."""
    h = x if residual is None else x + residual
    rstd = 1 / np.sqrt((h * h).mean(-1) + eps)
    y = h * rstd[..., None]
    return (y if w is None else y * w), h, rstd


def rmsnorm_grads(dy, h, w=None, dh=None, eps=1e-6):
    """(dx, dw)."""
    rstd = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    wdy = dy if w is None else dy * w
    dx = rstd * (wdy - h * rstd ** 2 * (wdy * h).mean(-1, keepdims=True))
    return (dx if dh is None else dx + dh), (dy * h * rstd).reshape(-1, h.shape[-1]).sum(0)


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, probability) of one row."""
    z = [-math.inf if math.isnan(x) else float(x) for x in z]
    top = max(z)
    if top == -math.inf:
        return -1, 0.0
    if temperature <= 0:
        return z.index(top), 1.0
    w = [1.0 if x == top else 0.0 if x == -math.inf or top == math.inf else math.exp((x - top) / temperature) for x in z]
    order = sorted(range(len(z)), key=lambda i: (-z[i], i))
    if 1 <= top_k < len(z):
        order = order[:top_k]
    if top_p < 1:
        total, kept, run = math.fsum(w[i] for i in order), [], 0.0
        for i in order:
            if kept and run >= top_p * total:
                break
            kept.append(i)
            run = math.fsum(w[j] for j in kept) if len(kept) < 200 else run + w[i]
        order = kept
    order = sorted(i for i in order if w[i] >= min_p or w[i] == 1.0)
    total, run, last = math.fsum(w[i] for i in order), 0.0, order[0]
    for i in order:
        run += w[i]
        if w[i] > 0:
            last = i
            if run > u * total:
                break
    return last, w[last] / total
