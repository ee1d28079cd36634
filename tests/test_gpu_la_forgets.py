"""What a linear attention forgets: everything in front of a step whose decay is zero, and nothing else.  Decays that together leave
nothing of a number multiply it: an infinity or NaN stays, and of a large number what is left of it, in every length of a
chunk, a segment or a stretch."""
import numpy as np
import pytest
import torch

import block_ref
import paper_2503_01868_amd as hy

from gpu_util import say

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def wide(t):
    return None if t is None else t.double().cpu().numpy()


def close(got, ref, size, dtype, what, steps, extra=0.0, least=2.0 ** -100):
    """`size` is the same sum with every term's magnitude.  fp32: 2e-5 of it for sums and for powers of two of up to 252, whose
    exponent is rounded to 2^-17 (2^-17 ln 2 = 5.3e-6, twice); a step taken by itself multiplies by the square of a power of
    two, whose last bit may be off and whose argument of at most 4 is rounded to 2^-23, and rounds twice: 2 (2^-23 + 2^-23 ln 2) + 2 x 2^-24
    = 5.3e-7, the same way at every step where decays are the same.  bf16: one rounding of a term, 2^-8, and one of the
    stored element.  What is below `least` is nothing."""
    got = wide(got)
    assert got.shape == ref.shape, what
    bound = (2e-5 + 5.3e-7 * steps) * size + extra + least
    if dtype == "bf16":
        bound = bound + 2.0 ** -8 * size + 2.0 ** -8 * np.abs(ref)
    fine = np.isfinite(ref)
    assert np.isfinite(got[fine]).all(), what
    worst = (np.abs(got - ref) - bound)[fine]
    assert not worst.size or worst.max() <= 0, (what, worst.max(), np.abs(ref[fine]).max())


def make(seed, B, L, H, dk, dv, dtype, decay):
    rng = np.random.default_rng(seed)

    def t(x, to=DTYPES[dtype]):
        return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(to).cuda()

    q, k = (t(rng.normal(size=(B, L, H, dk))) for _ in range(2))
    v, dy = (t(rng.normal(size=(B, L, H, dv))) for _ in range(2))
    state, dstate = (t(rng.normal(size=(B, H, dk, dv)), torch.float32) for _ in range(2))
    return q, k, v, t(np.full((B, L, H), decay)), dy, state, dstate


def pairs(q, k, size):
    """What the gradients of the log decays may be off by: they are sums of q . dq - k . dk over the steps of a chunk on one side of a
    decay, of which the pairs of steps that do not reach over it cancel, with the error of each, 2e-5 of its terms' magnitudes."""
    terms = (np.abs(wide(q)) * size[0]).sum(-1) + (np.abs(wide(k)) * size[1]).sum(-1)
    return 2e-5 * np.concatenate([np.broadcast_to(c.sum(1, keepdims=True), c.shape) for c in np.split(terms, range(64, terms.shape[1], 64), 1)], 1)


def stretches(q, k, v, g, state, lengths):
    """(y, state) of the sequence taken in stretches of these lengths in turn; a length of 0: single tokens from there on."""
    ys, at, i, L = [], 0, 0, q.shape[1]
    while at < L:
        n = lengths[i % len(lengths)]
        i += 1
        if n == 0:
            state = state.clone()
            ys += [hy.hyena_la_step(*(x[:, t].contiguous() for x in (q, k, v, g)), state, 0.5)[:, None] for t in range(at, L)]
            break
        y, state, _ = hy.hyena_la_fwd_carry(*(x[:, at:at + n] for x in (q, k, v, g)), 0.5, state_in=state)
        ys.append(y)
        at += n
    return torch.cat(ys, 1), state


CUTS = [(10 ** 6,), (64,), (1, 40, 100), (0,)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,dk,dv", [(150, 40, 72), (1100, 16, 48)])
@pytest.mark.parametrize("decay", [-0.5, -2.0, -60.0])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_until_a_reset(bad, decay, L, dk, dv, dtype):
    """One number of the first state is bad, and one of the last state's gradient: the column of y that it is in is not finite at any
    step, however the sequence is cut, nor is the number itself at the end; all others are as without it."""
    say("la bad state %s decay %g L=%d %s" % (bad, decay, L, dtype))
    q, k, v, g, dy, state, dstate = make(L, 1, L, 2, dk, dv, dtype, decay)
    w = [wide(x) for x in (q, k, v, g)]
    a = [abs(x) for x in w[:3]] + w[3:]
    ry, rs = block_ref.la(*w, 1, 0.5, wide(state))
    ay, as_ = block_ref.la(*a, 1, 0.5, abs(wide(state)))
    bad_in, bad_out = state.clone(), dstate.clone()
    bad_in[0, 1, 3, 5], bad_out[0, 1, 7, 11] = bad, bad
    ry[0, :, 1, 5], rs[0, 1, 3, 5] = np.nan, np.nan
    for cut in CUTS:
        y, s = stretches(q, k, v, g, bad_in, cut)
        close(y, ry, ay, dtype, "y %s" % (cut,), 100)
        close(s, rs, as_, "f32", "state %s" % (cut,), 100)
        assert not torch.isfinite(y[0, :, 1, 5]).any(), cut
        assert not torch.isfinite(s[0, 1, 3, 5]), cut
    ref = block_ref.la_grads(wide(dy), *w, 1, 0.5, wide(state), wide(dstate))
    size = block_ref.la_grads(abs(wide(dy)), *a, 1, 0.5, abs(wide(state)), abs(wide(dstate)))
    marks = hy.hyena_la_fwd_carry(q, k, v, g, 0.5, state_in=bad_in, want_marks=True)[2]
    for given in (marks, None):
        dq, dk_, dv_, dg, ds = hy.hyena_la_bwd(dy, q, k, v, g, 0.5, marks=given, state_in=bad_in, dstate_out=bad_out, want_dstate=True)
        for what, got, r, z, at in (("dq", dq, ref[0], size[0], np.s_[0, :, 1, 3]), ("dk", dk_, ref[1], size[1], np.s_[0, :, 1, 7]),
                                    ("dv", dv_, ref[2], size[2], np.s_[0, :, 1, 11]), ("dg", dg, ref[3], size[3], np.s_[0, :, 1]),
                                    ("dstate", ds, ref[4], size[4], np.s_[0, 1, 7, 11])):
            assert not np.isfinite(wide(got)[at]).any(), what
            r = r.copy()
            r[at] = np.nan
            close(got, r, z, "f32" if what == "dstate" else dtype, what, 100, extra=pairs(q, k, size) if what == "dg" else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,decay", [(64, -1.5), (150, -1.5), (150, -0.9), (700, -0.2)])
@pytest.mark.parametrize("alone", [False, True])
def test_a_large_state_leaves_what_is_left_of_it(alone, L, decay, dtype):
    """2^100 in every number of the first state of a head and of the last state's gradient of another; beside what the steps add, and
    where they add nothing."""
    say("la large state decay %g L=%d alone %s %s" % (decay, L, alone, dtype))
    q, k, v, g, dy, state, dstate = make(L, 1, L, 2, 24, 40, dtype, decay)
    if alone:
        v.zero_(), dy.zero_()
    state[:, 0] *= 2.0 ** 100
    dstate[:, 1] *= 2.0 ** 100
    w = [wide(x) for x in (q, k, v, g)]
    a = [abs(x) for x in w[:3]] + w[3:]
    ry, rs = block_ref.la(*w, 1, 0.5, wide(state))
    ay, as_ = block_ref.la(*a, 1, 0.5, abs(wide(state)))
    for cut in CUTS:
        y, s = stretches(q, k, v, g, state, cut)
        close(y, ry, ay, dtype, "y %s" % (cut,), L)
        close(s, rs, as_, "f32", "state %s" % (cut,), L)
    ref = block_ref.la_grads(wide(dy), *w, 1, 0.5, wide(state), wide(dstate))
    size = block_ref.la_grads(abs(wide(dy)), *a, 1, 0.5, abs(wide(state)), abs(wide(dstate)))
    # of <S, M>, what one of them holds below 2^-124 is nothing, however large the other is
    t, there = np.arange(L)[None, :, None], [abs(wide(x)).sum((2, 3))[:, None] for x in (state, dstate)]
    nothing = 2.0 ** -124 * (there[0] * np.exp(decay * t) + there[1] * np.exp(decay * (L - 1 - t)))
    marks = hy.hyena_la_fwd_carry(q, k, v, g, 0.5, state_in=state, want_marks=True)[2]
    for given in (marks, None):
        grads = hy.hyena_la_bwd(dy, q, k, v, g, 0.5, marks=given, state_in=state, dstate_out=dstate, want_dstate=True)
        for name, x, r, z in zip(("dq", "dk", "dv", "dg", "dstate"), grads, ref, size):
            close(x, r, z, "f32" if name == "dstate" else dtype, name, L, extra=pairs(q, k, size) + nothing if name == "dg" else 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_numbers_leave_what_is_left_of_them(dtype):
    """Products of 2^80 in the first steps, of which later steps with numbers of 2^40 see what decays of e^-1.9 a step leave, 2^-170 of
    them at the end of a chunk: products of three numbers that are far from nothing.  (A factor times one number may lose what is below
    2^-126, which is multiplied by another of less than 2^43 in 64 rows at most: 2^-77.)"""
    L, least = 64, 2.0 ** -77
    q, k, v, g, dy, _, _ = make(3, 1, L, 1, 16, 32, dtype, -1.9)
    for x, first in ((k, True), (v, True), (q, False), (dy, False)):
        x.clamp_(-4, 4)
        if first:
            x[:, 4:] = 0
            x[:, :4] *= 2.0 ** 40
        else:
            x[:, :30] = 0
            x[:, 30:] *= 2.0 ** 40
    w = [wide(x) for x in (q, k, v, g)]
    a = [abs(x) for x in w[:3]] + w[3:]
    ry, rs = block_ref.la(*w, 1, 1.0)
    ay, as_ = block_ref.la(*a, 1, 1.0)
    assert np.abs(ry[0, 50]).max() > 2.0 ** -30
    y, s, marks = hy.hyena_la_fwd_carry(q, k, v, g, want_marks=True)
    close(y, ry, ay, dtype, "y", L, least=least)
    close(s, rs, as_, "f32", "state", L, least=least)
    grads = hy.hyena_la_bwd(dy, q, k, v, g, marks=marks)
    ref, size = block_ref.la_grads(wide(dy), *w, 1, 1.0), block_ref.la_grads(abs(wide(dy)), *a, 1, 1.0)
    for name, x, r, z in zip(("dq", "dk", "dv", "dg"), grads, ref, size):
        close(x, r, z, dtype, name, L, extra=pairs(q, k, size) if name == "dg" else 0.0, least=least)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_numbers_beside_infinities(dtype):
    """Numbers of 2^100 in columns of a state (rows of its gradient) where others hold an infinity and NaN."""
    L, decay = 150, -0.9
    q, k, v, g, dy, state, dstate = make(5, 1, L, 1, 24, 40, dtype, decay)
    state[0, 0, :, 8] *= 2.0 ** 100
    dstate[0, 0, 9] *= 2.0 ** 100
    w = [wide(x) for x in (q, k, v, g)]
    a = [abs(x) for x in w[:3]] + w[3:]
    ry, rs = block_ref.la(*w, 1, 0.5, wide(state))
    ay, as_ = block_ref.la(*a, 1, 0.5, abs(wide(state)))
    ref = block_ref.la_grads(wide(dy), *w, 1, 0.5, wide(state), wide(dstate))
    size = block_ref.la_grads(abs(wide(dy)), *a, 1, 0.5, abs(wide(state)), abs(wide(dstate)))
    state[0, 0, 3, 5], state[0, 0, 4, 6] = float("inf"), float("nan")
    dstate[0, 0, 7, 11], dstate[0, 0, 8, 12] = -float("inf"), float("nan")
    ry[..., [5, 6]], rs[0, 0, 3, 5], rs[0, 0, 4, 6] = np.nan, np.nan, np.nan
    y, s, marks = hy.hyena_la_fwd_carry(q, k, v, g, 0.5, state_in=state, want_marks=True)
    close(y, ry, ay, dtype, "y", L)
    close(s, rs, as_, "f32", "state", L)
    grads = hy.hyena_la_bwd(dy, q, k, v, g, 0.5, marks=marks, dstate_out=dstate, want_dstate=True)
    for name, x, r, z, at in (("dq", grads[0], ref[0], size[0], [3, 4]), ("dk", grads[1], ref[1], size[1], [7, 8]), ("dv", grads[2], ref[2], size[2], [11, 12])):
        r = r.copy()
        r[..., at] = np.nan
        close(x, r, z, dtype, name, L)
        assert not np.isfinite(wide(x)[..., at]).any(), name
