"""Gated linear recurrence against its 64-bit form: sizes around the tiles, groups of every kind, both storage types, states in
and out, resets, views, and its single-token form."""
import numpy as np
import pytest
import torch

import model_ref
import paper_2503_01868_amd as hy
from paper_2503_01868_amd import binding

from gpu_util import say

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def close(got, ref, dtype, what):
    """fp32 arithmetic: 1e-5 of the largest value (the library's bar: some hundred roundings of 6e-8 add up); a stored bf16
    element besides: one rounding, 2^-8 of itself."""
    got = got.double().cpu().numpy()
    assert got.shape == ref.shape, what
    if ref.size == 0:
        return
    assert np.isfinite(got).all(), what
    bound = 1e-5 * np.abs(ref).max() + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0)
    worst = (np.abs(got - ref) - bound).max()
    assert worst <= 0, (what, worst)


def wide(t):
    return t.double().cpu().numpy()


def make(seed, B, L, D, group, dtype, resets=False):
    rng = np.random.default_rng(seed)

    def t(x, to=DTYPES[dtype]):
        return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(to).cuda()

    q, k, v, dy = (t(rng.normal(size=(B, L, D))) for _ in range(4))
    g = -np.exp(rng.uniform(np.log(1e-3), 0, size=(B, L, D // group)))
    if resets:
        g[rng.uniform(size=g.shape) < 0.05] = -np.inf
    state, dstate = (t(rng.normal(size=(B, D)), torch.float32) for _ in range(2))
    return q, k, v, t(g), dy, state, dstate


SHAPES = [(1, 1, 1, 1), (1, 2, 2, 1), (2, 1, 64, 1), (1, 8, 130, 1), (1, 63, 128, 16), (2, 64, 130, 2), (1, 65, 192, 3),
          (3, 200, 1000, 8), (1, 300, 7, 7), (2, 129, 256, 128), (1, 130, 512, 512), (1, 127, 96, 32), (1, 1100, 64, 4),
          (2, 511, 129, 1), (1, 140, 60, 6), (1, 70, 64, 64), (2, 66, 384, 192)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D,group", SHAPES)
def test_forward_and_gradients(B, L, D, group, dtype):
    say("glr B=%d L=%d D=%d group=%d %s" % (B, L, D, group, dtype))
    for carry in (False, True):
        q, k, v, g, dy, state, dstate = make(L + D, B, L, D, group, dtype, resets=carry)
        state, dstate = (state, dstate) if carry else (None, None)
        w = [wide(x) for x in (q, k, v, g)]
        s0 = None if state is None else wide(state)
        ry, rs, _ = model_ref.glr(*w, group, s0)
        y, s, marks = hy.hyena_glr_fwd_carry(q, k, v, g, group, state_in=state, want_state=True, want_marks=True)
        close(y, ry, dtype, "y")
        close(s, rs, "f32", "state")
        if not carry:
            assert torch.equal(hy.hyena_glr_fwd(q, k, v, g, group), y)
        ref = model_ref.glr_grads(wide(dy), *w, group, s0, None if dstate is None else wide(dstate))
        grads = hy.hyena_glr_bwd(dy, q, k, v, g, group, marks=marks, dstate_out=dstate, want_dstate=True)
        again = hy.hyena_glr_bwd(dy, q, k, v, g, group, state_in=state, dstate_out=dstate, want_dstate=True)
        for name, a, b, r in zip(("dq", "dk", "dv", "dg", "dstate"), grads, again, ref):
            close(a, r, "f32" if name == "dstate" else dtype, name)
            close(b, r, "f32" if name == "dstate" else dtype, name + " without marks")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_tiles_are_deterministic(dtype):
    """Enough tiles that they do not all run at once."""
    q, k, v, g, dy, state, dstate = make(5, 2, 20000, 192, 1, dtype)
    ry, rs, _ = model_ref.glr(*(wide(x) for x in (q, k, v, g)), 1, wide(state))
    outs = []
    for _ in range(3):
        y, s, marks = hy.hyena_glr_fwd_carry(q, k, v, g, 1, state_in=state, want_marks=True)
        outs.append((y, s) + hy.hyena_glr_bwd(dy, q, k, v, g, 1, marks=marks, dstate_out=dstate, want_dstate=True))
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            assert torch.equal(a, b)
    close(outs[0][0], ry, dtype, "y")
    close(outs[0][1], rs, "f32", "state")
    ref = model_ref.glr_grads(wide(dy), *(wide(x) for x in (q, k, v, g)), 1, wide(state), wide(dstate))
    for a, r, n in zip(outs[0][2:], ref, ("dq", "dk", "dv", "dg", "dstate")):
        close(a, r, "f32" if n == "dstate" else dtype, n)


@pytest.mark.parametrize("dtype,group", [("f32", 1), ("bf16", 16), ("bf16", 3)])
def test_tiles_that_do_not_wait_give_the_same_bits(dtype, group):
    q, k, v, g, dy, state, dstate = make(6, 2, 900, 192, group, dtype)

    def step():
        y, s, marks = hy.hyena_glr_fwd_carry(q, k, v, g, group, state_in=state, want_marks=True)
        return (y, s, marks) + hy.hyena_glr_bwd(dy, q, k, v, g, group, marks=marks, dstate_out=dstate, want_dstate=True)

    waited = step()
    binding.set_option("glr_wait", 1)
    try:
        alone = step()
    finally:
        binding.set_option("glr_wait", 0)
    for a, b in zip(waited, alone):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,D,group", [("bf16", 256, 1), ("bf16", 250, 5), ("f32", 128, 16)])
def test_stretches_and_single_tokens_continue_each_other(dtype, D, group):
    B, L = 2, 150
    q, k, v, g, _, state, _ = make(8, B, L, D, group, dtype)
    ry, rs, _ = model_ref.glr(*(wide(x) for x in (q, k, v, g)), group, wide(state))
    ys, s = [], state
    for lo, hi in ((0, 1), (1, 65), (65, 140)):
        y, s, _ = hy.hyena_glr_fwd_carry(*(x[:, lo:hi] for x in (q, k, v, g)), group, state_in=s)
        ys.append(y)
    for t in range(140, L):
        before = s
        ys.append(hy.hyena_glr_step(*(x[:, t].contiguous() for x in (q, k, v, g)), s, group)[:, None])
        assert s is before
    close(torch.cat(ys, 1), ry, dtype, "y")
    close(s, rs, "f32", "state")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 24])
def test_views_of_a_fused_projection_and_repeated_rows(dtype, D):
    """q, k, v as thirds of one [B, L, 3 D] tensor, a transposed [L, B, D] tensor, a gate that is the same at every step."""
    B, L = 3, 100
    q, k, v, g, dy, state, _ = make(11, B, L, D, 1, dtype)
    fused = torch.cat([q, k, v], 2)
    fq, fk, fv = fused.split(D, 2)
    tdy = dy.transpose(0, 1).contiguous().transpose(0, 1)
    same = g[:1, :1].expand(B, L, D)
    args = [wide(x) for x in (q, k, v)] + [wide(same)]
    y, s, marks = hy.hyena_glr_fwd_carry(fq, fk, fv, same, 1, state_in=state, want_marks=True)
    ry, rs, _ = model_ref.glr(*args, 1, wide(state))
    close(y, ry, dtype, "y")
    close(s, rs, "f32", "state")
    for n, a, r in zip(("dq", "dk", "dv", "dg"), hy.hyena_glr_bwd(tdy, fq, fk, fv, same, 1, marks=marks),
                       model_ref.glr_grads(wide(dy), *args, 1, wide(state))):
        close(a, r, dtype, n)


def test_odd_row_distances():
    """Rows that begin at odd elements, under an even width."""
    B, L, D = 1, 90, 32
    q, k, v, g, dy, _, _ = make(12, B, L, D, 1, "bf16")
    far = torch.zeros(B, L, D + 1, dtype=torch.bfloat16, device="cuda")
    far[:, :, :D] = k
    y = hy.hyena_glr_fwd(q, far[:, :, :D], v, g)
    assert torch.equal(y, hy.hyena_glr_fwd(q, k, v, g))


def test_no_steps_and_no_sequences():
    dev = "cuda"
    z = torch.empty(2, 0, 8, device=dev)
    state, d = torch.randn(2, 8, device=dev), torch.randn(2, 8, device=dev)
    y, s, marks = hy.hyena_glr_fwd_carry(z, z, z, z, state_in=state, want_marks=True)
    assert y.shape == z.shape and torch.equal(s, state) and marks.numel() == 0
    assert (hy.hyena_glr_fwd_carry(z, z, z, z)[1] == 0).all()
    grads = hy.hyena_glr_bwd(z, z, z, z, z, marks=marks, dstate_out=d, want_dstate=True)
    assert torch.equal(grads[4], d)
    e = torch.empty(0, 5, 8, device=dev)
    assert hy.hyena_glr_fwd(e, e, e, e).shape == e.shape
    e = torch.empty(0, 8, device=dev)
    assert hy.hyena_glr_step(e, e, e, e, torch.empty(0, 8, device=dev)).shape == e.shape


def test_a_value_that_is_not_finite_stays_in_its_channel_and_behind_its_step():
    B, L, D = 1, 200, 128
    q, k, v, g, _, _, _ = make(13, B, L, D, 1, "bf16")
    clean = hy.hyena_glr_fwd(q, k, v, g)
    k[0, 100, 5] = float("nan")
    y = hy.hyena_glr_fwd(q, k, v, g)
    bad = torch.zeros_like(y, dtype=torch.bool)
    bad[0, 100:, 5] = True
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[~bad])


def test_on_another_stream_with_a_workspace_of_the_caller():
    q, k, v, g, dy, _, _ = make(14, 1, 700, 256, 16, "bf16")
    want = hy.hyena_glr_fwd(q, k, v, g, 16)
    need = binding.lib().hyena_glr_fwd_workspace_bytes(1, 700, 256, 16, 1)
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(q)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    hy.hyena_glr_fwd(q, k, v, g, 16, out=out, workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(out, want)
    with pytest.raises(hy.HyenaError):
        hy.hyena_glr_fwd(q, k, v, g, 16, workspace=ws[:need - 1])


def test_inside_a_graph():
    """Replays see new inputs and give what eager calls give."""
    q, k, v, g, dy, state, dstate = make(15, 1, 1000, 256, 16, "bf16")

    def step():
        y, s, marks = hy.hyena_glr_fwd_carry(q, k, v, g, 16, state_in=state, want_marks=True)
        return (y, s) + hy.hyena_glr_bwd(dy, q, k, v, g, 16, marks=marks, dstate_out=dstate, want_dstate=True)

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        step()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(4):
        k.copy_(torch.randn_like(k))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)


def test_refusals():
    q, k, v, g, dy, state, _ = make(16, 2, 10, 16, 4, "bf16")
    with pytest.raises(ValueError):
        hy.hyena_glr_fwd(q, k.float(), v, g, 4)
    with pytest.raises(ValueError):
        hy.hyena_glr_fwd(q, k, v, g, 2)
    with pytest.raises(ValueError):
        hy.hyena_glr_fwd(q, k, v, g, 3)
    with pytest.raises(ValueError):
        hy.hyena_glr_fwd(q.cpu(), k, v, g, 4)
    with pytest.raises(ValueError):
        hy.hyena_glr_fwd(q.transpose(1, 2).contiguous().transpose(1, 2), k, v, g, 4)
    with pytest.raises(TypeError):
        hy.hyena_glr_fwd(q.half(), k.half(), v.half(), g.half(), 4)
    with pytest.raises(ValueError):
        hy.hyena_glr_fwd_carry(q, k, v, g, 4, state_in=state.bfloat16())
    with pytest.raises(ValueError):
        hy.hyena_glr_bwd(dy, q, k, v, g, 4, marks=state)
    with pytest.raises(hy.HyenaError):
        hy.hyena_glr_fwd(q, k, v, g, 4, out=q)
    with pytest.raises(ValueError):
        hy.hyena_glr_step(q[:, 0], k[:, 0], v[:, 0], g[:, 0], state, 4)


def test_a_token_inside_a_graph():
    """A decoder's step captured once: every replay takes the state one token further, as eager calls do."""
    q, k, v, g, _, _, _ = make(21, 4, 1, 256, 16, "bf16")
    q, k, v, g = (t[:, 0].contiguous() for t in (q, k, v, g))
    state = torch.zeros(4, 256, device="cuda")
    other = state.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        hy.hyena_glr_step(q, k, v, g, state, 16)
    side.synchronize()
    state.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = hy.hyena_glr_step(q, k, v, g, state, 16)
    for i in range(4):
        k.copy_(torch.randn_like(k))
        eager = hy.hyena_glr_step(q, k, v, g, other, 16)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager) and torch.equal(state, other)
