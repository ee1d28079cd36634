"""Host-only checks of linear attention, the norm and the choice of tokens: bad arguments are rejected before the GPU is touched."""
import ctypes

import pytest

from paper_2503_01868_amd import binding

P = [ctypes.c_void_p(1 << 20 | i << 36) for i in range(1, 20)]  # far apart, aligned, never looked at


def fwd(q=P[0], k=P[1], v=P[2], g=P[3], s_in=None, y=P[4], s_out=None, marks=None, strides=None, ws=P[5], nbytes=1 << 34, B=1, L=1000,
        H=4, group=1, dk=64, dv=64, scale=1.0, dtype=1):
    return binding.lib().hyena_la_fwd(q, k, v, g, s_in, y, s_out, marks, strides, ws, nbytes, B, L, H, group, dk, dv, scale, dtype, None)


def bwd(dy=P[0], q=P[1], k=P[2], v=P[3], g=P[4], marks=P[5], s_in=None, ds=None, dq=P[6], dk_=P[7], dv_=P[8], dg=P[9], ds_in=None,
        strides=None, ws=P[10], nbytes=1 << 34, B=1, L=1000, H=4, group=1, dk=64, dv=64, scale=1.0, dtype=1):
    return binding.lib().hyena_la_bwd(dy, q, k, v, g, marks, s_in, ds, dq, dk_, dv_, dg, ds_in, strides, ws, nbytes, B, L, H, group,
                                      dk, dv, scale, dtype, None)


def step(q=P[0], k=P[1], v=P[2], g=P[3], state=P[4], y=P[5], B=1, H=4, group=1, dk=64, dv=64, scale=1.0, dtype=1):
    return binding.lib().hyena_la_step(q, k, v, g, state, y, B, H, group, dk, dv, scale, dtype, None)


@pytest.mark.parametrize("call,names,outputs", [(fwd, "q k v g y", "y"), (bwd, "dy q k v g dq dk_ dv_ dg", "dq dk_ dv_ dg"),
                                                (step, "q k v g state y", "state y")])
def test_linear_attention_rejects_bad_arguments(call, names, outputs):
    for n in names.split():
        assert call(**{n: None}) == 1, n
        assert call(**{n: ctypes.c_void_p((1 << 40) + 1)}) == 4, n
    for n in outputs.split():  # inputs may begin at any element
        assert call(**{n: ctypes.c_void_p((1 << 40) + 8)}) == 4, n
    for n in ("B", "H") if call is step else ("B", "L", "H"):
        assert call(**{n: -1}) == 2, n
    for n in ("dk", "dv"):
        assert call(**{n: 0}) == 2 and call(**{n: -1}) == 2, n
    assert call(group=0) == 2 and call(group=3) == 2
    assert call(dtype=2) == 3 and call(dtype=-1) == 3
    assert call(B=1 << 40, H=1 << 40) == 2 and call(dk=1 << 40, dv=1 << 40) == 2
    assert call(dk=129 if call is not step else 65537) == 5 and call(B=1 << 22) == 5


def test_linear_attention_rejects_overlaps_strides_and_workspaces():
    assert fwd(y=P[0]) == 4 and fwd(s_out=P[4]) == 4 and fwd(marks=P[1]) == 4 and fwd(s_in=P[6], s_out=P[6]) == 4
    assert bwd(dq=P[0]) == 4 and bwd(dq=P[7]) == 4 and bwd(ds_in=P[5]) == 4 and bwd(dk_=P[3]) == 4
    assert step(state=P[0]) == 4 and step(y=P[4]) == 4
    assert fwd(nbytes=-1) == 2 and bwd(nbytes=-1) == 2
    assert fwd(ws=None) == 1 and fwd(nbytes=16) == 2 and fwd(ws=P[4]) == 4
    assert bwd(ws=None) == 1 and bwd(nbytes=16) == 2 and bwd(ws=P[9]) == 4
    n = 11
    assert fwd(strides=(ctypes.c_int64 * n)(0, -1)) == 2 and fwd(strides=(ctypes.c_int64 * n)(0, 1 << 60)) == 2
    assert bwd(strides=(ctypes.c_int64 * 14)(0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, -1)) == 2
    far = ((P[4].value - P[0].value) // 2 // 999) + 1  # rows of q reach as far as y
    assert fwd(strides=(ctypes.c_int64 * n)(0, far, 64, 0, 256, 64, 0, 256, 64, 0, 4)) == 4


def test_linear_attention_takes_empty_problems():
    assert fwd(B=0) == 0 and fwd(L=0) == 0 and fwd(H=0, q=None, y=None) == 0
    assert bwd(B=0, dy=None) == 0 and bwd(L=0) == 0
    assert step(B=0, q=None) == 0 and step(H=0) == 0


def test_linear_attention_sizes_its_buffers():
    lb = binding.lib()
    f, b, m = lb.hyena_la_fwd_workspace_bytes, lb.hyena_la_bwd_workspace_bytes, lb.hyena_la_marks_bytes
    assert f(1, 0, 4, 1, 64, 64, 1) == 0 == b(0, 10, 4, 1, 64, 64, 1, 1) == m(1, 0, 4, 1, 64, 64, 1)
    for bad in ((-1, 10, 4, 1, 64, 64, 1), (1, 10, 4, 3, 64, 64, 1), (1, 10, 4, 1, 64, 64, 7), (1, 10, 4, 1, 129, 64, 1)):
        assert f(*bad) == -1 and m(*bad) == -1 and b(*bad, 0) == -1
    assert f(1, 64, 4, 1, 64, 64, 1) == 0                                    # a chunk needs none
    assert 0 < m(1, 8192, 32, 1, 128, 128, 1) < 1 << 28
    assert b(1, 8192, 32, 1, 128, 128, 1, 0) >= b(1, 8192, 32, 1, 128, 128, 1, 1) + m(1, 8192, 32, 1, 128, 128, 1)
    assert b(1, 1000, 4, 2, 64, 64, 1, 1) > b(1, 1000, 4, 1, 64, 64, 1, 1)   # the heads' shares


def norm(x=P[0], r=P[1], w=P[2], y=P[3], y_scale=None, h=P[4], rstd=P[5], N=100, D=64, xs=64, rs=64, eps=1e-6, dtype=1):
    return binding.lib().hyena_rmsnorm_fwd(x, r, w, y, y_scale, h, rstd, N, D, xs, rs, eps, dtype, None)


def norm_bwd(dy=P[0], h=P[1], rstd=P[2], w=P[3], dh=P[4], dx=P[5], dw=P[6], ws=P[7], nbytes=1 << 30, N=100, D=64, dtype=1):
    return binding.lib().hyena_rmsnorm_bwd(dy, h, rstd, w, dh, dx, dw, ws, nbytes, N, D, dtype, None)


def test_the_norm_rejects_bad_arguments():
    for n in ("x", "y"):
        assert norm(**{n: None}) == 1, n
    for n in ("x", "r", "w", "y", "h"):
        assert norm(**{n: ctypes.c_void_p((1 << 41) + 1)}) == 4, n
    for n in ("rstd", "y_scale"):
        assert norm(**{n: ctypes.c_void_p((1 << 41) + 2)}) == 4, n
    assert norm(N=-1) == 2 and norm(D=0) == 2 and norm(xs=-1) == 2 and norm(rs=-1) == 2 and norm(N=1 << 40, D=1 << 40) == 2
    assert norm(xs=1 << 60) == 2 and norm(eps=-1.0) == 2 and norm(eps=float("nan")) == 2 and norm(r=None) == 2  # a sum of nothing
    assert norm(dtype=2) == 3 and norm(D=1 << 32) == 5
    assert norm(y=P[0]) == 4 and norm(y=P[4]) == 4 and norm(rstd=P[3]) == 4 and norm(h=P[2]) == 4 and norm(y_scale=P[5]) == 4
    assert norm(h=ctypes.c_void_p(P[1].value + 128)) == 4          # in place, but not the same rows
    assert norm(h=P[1], rs=128) == 4 and norm(h=P[1], rs=0) == 4   # in place on rows that are not dense
    assert norm(N=0, x=None, y=None) == 0


def test_the_gradient_of_the_norm_rejects_bad_arguments():
    for n in ("dy", "h", "rstd", "dx"):
        assert norm_bwd(**{n: None}) == 1, n
    for n in ("dy", "h", "w", "dh", "dx", "dw"):
        assert norm_bwd(**{n: ctypes.c_void_p((1 << 41) + 1)}) == 4, n
    assert norm_bwd(N=-1) == 2 and norm_bwd(D=0) == 2 and norm_bwd(w=None) == 2 and norm_bwd(dtype=2) == 3
    assert norm_bwd(dx=P[1]) == 4 and norm_bwd(dw=P[3]) == 4 and norm_bwd(dx=P[6]) == 4 and norm_bwd(dx=ctypes.c_void_p(P[0].value + 128)) == 4
    assert norm_bwd(ws=None) == 1 and norm_bwd(nbytes=16) == 2 and norm_bwd(nbytes=-1) == 2 and norm_bwd(ws=P[5]) == 4
    assert norm_bwd(ws=ctypes.c_void_p((1 << 41) + 8)) == 4
    assert norm_bwd(N=0, dy=None, dw=None, w=None, ws=None) == 0
    size = binding.lib().hyena_rmsnorm_bwd_workspace_bytes
    assert size(-1, 64, 1) == -1 and size(100, 0, 1) == -1 and size(100, 64, 1) == 100 * 64 * 4 and size(1 << 20, 4096, 1) < 1 << 24


def sample(z=P[0], u=P[1], t=P[2], k=P[3], p=P[4], m=P[5], token=P[6], prob=P[7], N=10, V=100, stride=100, dtype=1):
    return binding.lib().hyena_sample(z, u, t, 1.0, k, 0, p, 1.0, m, 0.0, token, prob, N, V, stride, dtype, None)


def test_the_choice_of_tokens_rejects_bad_arguments():
    for n in ("z", "u", "token"):
        assert sample(**{n: None}) == 1, n
    assert sample(z=ctypes.c_void_p((1 << 41) + 1)) == 4 and sample(token=ctypes.c_void_p((1 << 41) + 4)) == 4
    for n in ("u", "t", "k", "p", "m", "prob"):
        assert sample(**{n: ctypes.c_void_p((1 << 41) + 2)}) == 4, n
    assert sample(N=-1) == 2 and sample(V=0) == 2 and sample(stride=-1) == 2 and sample(stride=1 << 60) == 2 and sample(N=1 << 40, V=1 << 40) == 2
    assert sample(dtype=2) == 3 and sample(V=(1 << 22) + 1) == 5 and sample(N=(1 << 22) + 1) == 5
    assert sample(token=P[0]) == 4 and sample(prob=P[6]) == 4 and sample(prob=P[1]) == 4 and sample(token=P[3]) == 4
    assert sample(N=0, z=None, u=None) == 0
