"""The operators around the mixers in 64 bits, written out step by step (numpy)."""
import numpy as np


def glr(q, k, v, g, group=1, state=None):
    """(y, state after the last step, states after every step)."""
    B, L, D = q.shape
    a = np.exp(np.repeat(g, group, axis=2))
    s = np.zeros((B, D)) if state is None else state.astype(np.float64).copy()
    every = np.empty((B, L, D))
    for t in range(L):
        s = a[:, t] * s + k[:, t] * v[:, t]
        every[:, t] = s
    return q * every, s, every


def glr_grads(dy, q, k, v, g, group=1, state=None, dstate=None):
    """(dq, dk, dv, dg, dstate_in)."""
    B, L, D = q.shape
    a = np.exp(np.repeat(g, group, axis=2))
    _, _, every = glr(q, k, v, g, group, state)
    c = np.zeros((B, D)) if dstate is None else dstate.astype(np.float64).copy()
    dq, dk, dv, da = (np.zeros((B, L, D)) for _ in range(4))
    for t in range(L - 1, -1, -1):
        before = every[:, t - 1] if t > 0 else (np.zeros((B, D)) if state is None else state)
        m = q[:, t] * dy[:, t] + c
        dq[:, t], dk[:, t], dv[:, t] = dy[:, t] * every[:, t], m * v[:, t], m * k[:, t]
        c = a[:, t] * m
        da[:, t] = c * before
    return dq, dk, dv, da.reshape(B, L, D // group, group).sum(3), c


def adamw(p, g, m, v, lr, step, decay=0.0, beta1=0.9, beta2=0.95, eps=1e-8, scale=1.0):
    """(p, m, v) after the step."""
    g = g * scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p - lr * decay * p - lr * (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps), m, v


def xent(x, w, target):
    """(loss, lse, z); rows whose target is no row of w have loss 0."""
    z = x @ w.T
    top = z.max(1, keepdims=True)
    lse = (top + np.log(np.exp(z - top).sum(1, keepdims=True)))[:, 0]
    counts = (target >= 0) & (target < len(w))
    loss = np.where(counts, lse - z[np.arange(len(x)), np.where(counts, target, 0)], 0.0)
    return loss, lse, z


def xent_grads(dloss, x, w, target):
    """(dx, dw)."""
    _, lse, z = xent(x, w, target)
    counts = (target >= 0) & (target < len(w))
    p = np.exp(z - lse[:, None])
    p[np.flatnonzero(counts), target[counts]] -= 1
    p *= np.where(counts, dloss, 0.0)[:, None]
    return p @ w, p.T @ x
