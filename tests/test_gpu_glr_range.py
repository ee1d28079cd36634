"""Gated linear recurrence over the whole range of its gates: decays whose product passes the range of fp32 while the states stay
within it, growth that a reset ends, resets that forget what is not finite, and tiles that come by their edge in different ways."""
import numpy as np
import pytest
import torch

import model_ref
import paper_2503_01868_amd as hy
from paper_2503_01868_amd import binding

from gpu_util import say

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SHAPES = [(1, 1100, 64, 1), (2, 1100, 256, 1), (1, 1100, 258, 1), (1, 1100, 320, 64), (1, 1100, 21, 3)]
NAMES = ("dq", "dk", "dv", "dg", "dstate")


def wide(t):
    return t.double().cpu().numpy()


def tensor(x, dtype):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(DTYPES[dtype]).cuda()


def inputs(seed, B, L, D, g, scale, dtype):
    """q of order 1, k v and dy of order `scale`; g as [B, L, D / group]."""
    rng = np.random.default_rng(seed)
    root = np.sqrt(scale)
    q, k, v, dy = (rng.normal(size=(B, L, D)) * f for f in (1.0, root, root, scale))
    return tuple(tensor(x, dtype) for x in (q, k, v, g, dy))


def close(got, ref, mass, rel, dtype, what):
    """`rel` of the sum of magnitudes that went into an element; a stored bf16 element besides, 2^-8 of itself; 1e-36: numbers
    that fp32 holds with fewer bits."""
    got = wide(got)
    assert np.isfinite(got).all(), (what, int((~np.isfinite(got)).sum()))
    worst = (np.abs(got - ref) - (rel * mass + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0) + 1e-36)).max()
    assert worst <= 0, (what, worst)


def check(q, k, v, g, dy, group, dtype):
    """Against the 64-bit form.  A step's decay is off by (2 + |g|) 2^-24 and its product and sum by 2^-24 each; a stretch's
    decay is the exponential of a sum of at most 24 terms in a row, off by 24 roundings of the sum of |g|, and of a few besides, in
    each of three ways to a state (waves, tiles, blocks): 2^-24 (8 L + 40 sum |g|) of the magnitudes, twice for a product of both."""
    L = q.shape[1]
    w = [wide(x) for x in (q, k, v, g)]
    total = np.abs(np.where(np.isfinite(w[3]) & (w[3] > -1e3), w[3], 0.0)).sum(1).max()
    rel = 2.0 ** -24 * (8 * L + 40 * total)
    a = [np.abs(x) for x in w[:3]] + [w[3]]
    ry, rs, _ = model_ref.glr(*w, group)
    my, ms, _ = model_ref.glr(*a, group)
    y, s, marks = hy.hyena_glr_fwd_carry(q, k, v, g, group, want_marks=True)
    close(y, ry, my, rel, dtype, "y")
    close(s, rs, ms, rel, "f32", "state")
    ref = model_ref.glr_grads(wide(dy), *w, group)
    mass = model_ref.glr_grads(np.abs(wide(dy)), *a, group)
    for marked in (marks, None):
        got = hy.hyena_glr_bwd(dy, q, k, v, g, group, marks=marked, want_dstate=True)
        for n, x, r, m in zip(NAMES, got, ref, mass):
            close(x, r, m, 2 * rel, "f32" if n == "dstate" else dtype, n)
    return y, s, got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D,group", SHAPES)
def test_nothing_grows_from_nothing(B, L, D, group, dtype):
    """k v = 0 and dy = 0 under a growth that passes any range: zeros."""
    say("glr zeros B=%d L=%d D=%d group=%d %s" % (B, L, D, group, dtype))
    q, k, v, g, dy = inputs(1, B, L, D, np.full((B, L, D // group), 0.5), 1.0, dtype)
    k, dy = torch.zeros_like(k), torch.zeros_like(dy)
    y, s, marks = hy.hyena_glr_fwd_carry(q, k, v, g, group, want_marks=True)
    assert (y == 0).all() and (s == 0).all() and (marks == 0).all()
    for n, x in zip(NAMES, hy.hyena_glr_bwd(dy, q, k, v, g, group, marks=marks, want_dstate=True)):
        assert (x == 0).all(), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D,group", SHAPES)
def test_growth_of_small_states_that_a_reset_ends(B, L, D, group, dtype):
    """1e-20 e^120 at the most, under decays whose product over 512 steps is e^102."""
    say("glr growth B=%d L=%d D=%d group=%d %s" % (B, L, D, group, dtype))
    g = np.full((B, L, D // group), 0.2)
    g[:, 600] = -np.inf
    check(*inputs(2, B, L, D, g, 1e-20, dtype), group, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,group", [(64, 1), (256, 1), (320, 64), (21, 3)])
def test_growth_and_decay_in_turn(D, group, dtype):
    """e^60 and e^-60 step by step: no product of a step's neighbours tells how far the states have come."""
    say("glr turns D=%d group=%d %s" % (D, group, dtype))
    L = 300
    g = np.where(np.arange(L) % 2 == 0, 60.0, -60.0)[None, :, None].repeat(D // group, 2)
    check(*inputs(3, 1, L, D, g, 1.0, dtype), group, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_reset_in_front_of_growth_and_behind_it(dtype):
    """Ordinary values around resets, in tiles and blocks of every kind; mild growth in between (e^26 at the most)."""
    rng = np.random.default_rng(4)
    L, D = 1400, 64
    g = np.full((1, L, D), 0.5)
    g[rng.uniform(size=g.shape) < 0.5] = -0.5
    g[:, ::52] = -np.inf
    check(*inputs(4, 1, L, D, g, 1.0, dtype), 1, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D,group", [(64, 1), (256, 1), (320, 64), (21, 3)])
def test_a_reset_forgets_what_is_not_finite(D, group, bad, dtype):
    """In k of a document, in its gates and in the state before it: the next document has the bits that it has alone; a gradient that
    is not finite does not reach the document before."""
    say("glr forgets D=%d group=%d %s %s" % (D, group, bad, dtype))
    B, L, cut = 1, 1200, 700
    rng = np.random.default_rng(5)
    g = -np.exp(rng.uniform(np.log(1e-3), 0, size=(B, L, D // group)))
    g[:, 0] = g[:, cut] = -np.inf
    q, k, v, g, dy = inputs(5, B, L, D, g, 1.0, dtype)
    y, s, _ = hy.hyena_glr_fwd_carry(q, k, v, g, group)
    clean = hy.hyena_glr_bwd(dy, q, k, v, g, group, want_dstate=True)
    state = torch.full((B, D), bad, device="cuda")
    other = hy.hyena_glr_fwd_carry(q, k, v, g, group, state_in=state)
    assert torch.equal(other[0], y) and torch.equal(other[1], s)
    for at in (3, 690):
        k2, g2, dy2 = k.clone(), g.clone(), dy.clone()
        k2[:, at] = bad
        g2[:, at + 2] = bad
        y2, s2, marks = hy.hyena_glr_fwd_carry(q, k2, v, g2, group, want_marks=True)
        assert torch.equal(y2[:, cut:], y[:, cut:]) and torch.equal(s2, s)
        assert not torch.isfinite(y2[:, at]).any() and not torch.isfinite(y2[:, at + 3:cut]).any()
        assert torch.equal(y2[:, :at], y[:, :at])
        dy2[:, cut + 5] = bad
        got = hy.hyena_glr_bwd(dy2, q, k, v, g, group, want_dstate=True)
        for n, a, b in zip(NAMES[1:4], got[1:4], clean[1:4]):
            assert torch.equal(a[:, :cut], b[:, :cut]), n
            assert not torch.isfinite(a[:, cut + 1:cut + 5]).any(), n
        assert torch.equal(got[0][:, :cut], clean[0][:, :cut]) and torch.equal(got[4], clean[4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_lowest_number_is_a_reset(dtype):
    B, L, D = 2, 700, 128
    rng = np.random.default_rng(6)
    g = -np.exp(rng.uniform(np.log(1e-3), 0, size=(B, L, D)))
    g[rng.uniform(size=g.shape) < 0.01] = -np.inf
    q, k, v, g, dy = inputs(6, B, L, D, g, 1.0, dtype)
    low = torch.where(torch.isinf(g), torch.finfo(g.dtype).min, g)
    outs = []
    for gates in (g, low):
        y, s, marks = hy.hyena_glr_fwd_carry(q, k, v, gates, want_marks=True)
        outs.append((y, s) + hy.hyena_glr_bwd(dy, q, k, v, gates, marks=marks, want_dstate=True))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,D,group", [("bf16", 256, 1), ("bf16", 250, 5), ("f32", 128, 16)])
def test_single_tokens_take_growth_and_resets_like_stretches(dtype, D, group):
    """The bound of `check`, for two ways to the same state."""
    B, L, start = 2, 660, 560
    g = np.full((B, L, D // group), 0.2)
    g[:, 630] = -np.inf
    q, k, v, g, _ = inputs(7, B, L, D, g, 1e-20, dtype)
    y, s, _ = hy.hyena_glr_fwd_carry(q, k, v, g, group)
    mass = model_ref.glr(*(np.abs(wide(x)) for x in (q, k, v)), wide(g), group)
    rel = 2.0 ** -24 * (8 * L + 40 * 0.21 * L)
    state = hy.hyena_glr_fwd_carry(*(x[:, :start] for x in (q, k, v, g)), group)[1]
    for t in range(start, L):
        one = hy.hyena_glr_step(*(x[:, t].contiguous() for x in (q, k, v, g)), state, group)
        close(one, wide(y[:, t]), mass[0][:, t], 2 * rel, dtype, t)
    close(state, wide(s), mass[1], 2 * rel, "f32", "state")
    bad = torch.full((B, D), float("nan"), device="cuda")
    reset = [x[:, 630].contiguous() for x in (q, k, v, g)]
    assert torch.equal(hy.hyena_glr_step(*reset, bad, group), y[:, 630]) and torch.isfinite(bad).all()


@pytest.mark.parametrize("dtype,D,group", [("f32", 192, 1), ("bf16", 192, 1), ("bf16", 256, 16)])
def test_tiles_that_find_their_edge_and_tiles_that_walk_give_the_same_bits(dtype, D, group):
    """Looking once, some workgroups of a long sequence find the state before them and others sum the sequence up."""
    B, L = 2, 12000
    rng = np.random.default_rng(8)
    g = -np.exp(rng.uniform(np.log(1e-3), 0, size=(B, L, D // group)))
    g[rng.uniform(size=g.shape) < 1e-3] = -np.inf
    g[:, 5000:5600] = 0.1
    q, k, v, g, dy = inputs(8, B, L, D, g, 1e-6, dtype)

    def step():
        y, s, marks = hy.hyena_glr_fwd_carry(q, k, v, g, group, want_marks=True)
        return (y, s, marks) + hy.hyena_glr_bwd(dy, q, k, v, g, group, marks=marks, want_dstate=True)

    waited = step()
    assert all(torch.isfinite(x).all() for x in waited)
    for how in (2, 2, 1):
        binding.set_option("glr_wait", how)
        try:
            other = step()
        finally:
            binding.set_option("glr_wait", 0)
        for a, b in zip(waited, other):
            assert torch.equal(a, b)
