"""Linear attention with decays against its 64-bit form: sizes around the chunks and tiles, shared heads, both storage types, states
in and out, resets, growth, what is not finite, views, and its single-token form."""
import numpy as np
import pytest
import torch

import block_ref
import paper_2503_01868_amd as hy

from gpu_util import say

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def close(got, ref, size, dtype, what, mixed=True, extra=0.0):
    """`size` is the same sum with every term's magnitude.  fp32 arithmetic: 2e-5 of it (some 300 roundings of 6e-8 in a row, and
    exponents of up to 126 whose last bit is worth 5e-6).  bf16: a term passes one rounding to bf16 (of A, or of a state where it
    is multiplied), 2^-8 of itself, and the stored element another."""
    got = got.double().cpu().numpy()
    assert got.shape == ref.shape, what
    if ref.size == 0:
        return
    bound = 2e-5 * size + extra + 1e-30
    if dtype == "bf16":
        bound = bound + (2.0 ** -8 * size if mixed else 0.0) + 2.0 ** -8 * np.abs(ref)
    fine = np.isfinite(ref)
    assert np.isfinite(got[fine]).all(), what
    worst = (np.abs(got - ref) - bound)[fine]
    assert not worst.size or worst.max() <= 0, (what, worst.max(), np.abs(ref).max())


def wide(t):
    return None if t is None else t.double().cpu().numpy()


def make(seed, B, L, H, group, dk, dv, dtype, resets=0.0, states=True):
    rng = np.random.default_rng(seed)

    def t(x, to=DTYPES[dtype]):
        return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(to).cuda()

    q, k = (t(rng.normal(size=(B, L, H // group, dk))) for _ in range(2))
    v, dy = (t(rng.normal(size=(B, L, H, dv))) for _ in range(2))
    g = -np.exp(rng.uniform(np.log(1e-3), 0.5, size=(B, L, H)))
    g[rng.uniform(size=g.shape) < resets] = -np.inf
    state, dstate = (t(rng.normal(size=(B, H, dk, dv)), torch.float32) for _ in range(2))
    return (q, k, v, t(g), dy) + ((state, dstate) if states else (None, None))


def check(q, k, v, g, dy, state, dstate, scale, dtype, marks_too=True):
    group = v.shape[2] // q.shape[2]
    w = [wide(x) for x in (q, k, v, g)]
    a = [abs(x) for x in w[:3]] + w[3:]
    s0, ds = wide(state), wide(dstate)
    sizes = None if s0 is None else abs(s0), None if ds is None else abs(ds)
    ry, rs = block_ref.la(*w, group, scale, s0)
    ay, as_ = block_ref.la(*a, group, scale, sizes[0])
    y, s, marks = hy.hyena_la_fwd_carry(q, k, v, g, scale, state_in=state, want_marks=True)
    close(y, ry, ay, dtype, "y")
    close(s, rs, as_, "f32", "state")
    if state is None:
        assert torch.equal(hy.hyena_la_fwd(q, k, v, g, scale), y)
    ref = block_ref.la_grads(wide(dy), *w, group, scale, s0, ds)
    size = block_ref.la_grads(abs(wide(dy)), *a, group, scale, *sizes)
    for given in (marks, None) if marks_too else (marks,):
        grads = hy.hyena_la_bwd(dy, q, k, v, g, scale, marks=given, state_in=state, dstate_out=dstate, want_dstate=True)
        for name, x, r, z in zip(("dq", "dk", "dv", "dg", "dstate"), grads, ref, size):
            # dg is made from sums over all pairs of a chunk, of which those that do not reach over its step cancel
            extra = 2e-5 * z.max() if name == "dg" and z.size else 0.0
            close(x, r, z, "f32" if name == "dstate" else dtype, name, extra=extra)


# B, L, H, group, dk, dv
SHAPES = [(1, 1, 1, 1, 1, 1), (2, 2, 3, 3, 8, 16), (1, 15, 2, 1, 33, 40), (1, 16, 2, 2, 64, 64), (3, 17, 4, 2, 40, 72), (1, 31, 1, 1, 16, 128),
          (1, 32, 2, 1, 65, 64), (2, 33, 2, 1, 128, 65), (1, 63, 2, 1, 128, 128), (1, 64, 4, 4, 64, 128), (2, 65, 2, 1, 128, 64),
          (1, 127, 3, 1, 100, 129), (1, 128, 2, 2, 24, 256), (1, 129, 2, 1, 64, 200), (1, 700, 2, 1, 128, 128), (2, 1000, 2, 2, 64, 72),
          (1, 1537, 1, 1, 48, 130), (1, 600, 1, 1, 7, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,H,group,dk,dv", SHAPES)
def test_forward_and_gradients(B, L, H, group, dk, dv, dtype):
    say("la B=%d L=%d H=%d group=%d dk=%d dv=%d %s" % (B, L, H, group, dk, dv, dtype))
    check(*make(L + dk, B, L, H, group, dk, dv, dtype, states=False), dk ** -0.5, dtype)
    check(*make(L + dk + 1, B, L, H, group, dk, dv, dtype, resets=0.03), 1.0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["slow", "fast", "still", "growing", "near the end of exp", "every step resets"])
def test_decays_of_every_kind(dtype, what):
    """Time constants far longer than the sequence, decays that leave nothing within a few steps, none at all, growth by e^70 over the
    sequence, log decays on both sides of -87.3."""
    B, L, H, dk, dv = 1, 330, 2, 32, 48
    q, k, v, g, dy, state, dstate = make(4, B, L, H, 1, dk, dv, dtype)
    rng = np.random.default_rng(5)
    new = {"slow": -1e-6 * rng.uniform(size=g.shape), "fast": -20 * rng.uniform(size=g.shape), "still": np.zeros(g.shape),
           "growing": 0.2 * rng.uniform(0.5, 1.5, size=g.shape), "near the end of exp": rng.choice([-0.01, -80.0, -87.0, -90.0, -1e30], size=g.shape),
           "every step resets": np.full(g.shape, -np.inf)}[what]
    g = torch.from_numpy(new.astype(np.float32)).to(g.dtype).cuda()
    check(q, k, v, g, dy, state, dstate, 0.2, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_growth_from_nothing_is_nothing(dtype):
    """e^(2 * 64) overflows; a state of zero stays zero under it."""
    q, k, v, g, dy, _, _ = make(4, 1, 200, 1, 1, 16, 16, dtype)
    g = torch.full_like(g, 2.0)
    k[:, :190] = 0
    y, s, marks = hy.hyena_la_fwd_carry(q, k, v, g, want_marks=True)
    w = [wide(x) for x in (q, k, v, g)]
    ry, rs = block_ref.la(*w)
    ay, as_ = block_ref.la(*[abs(x) for x in w])
    assert torch.equal(y[:, :190], torch.zeros_like(y[:, :190]))
    close(y, ry, ay, dtype, "y")
    close(s, rs, as_, "f32", "state")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_document_and_behind_its_step(dtype, bad):
    """Three documents in a row; one number of the second is bad in turn of k, v, q, dy, g: whatever does not depend on it has the
    values that it has without it (to rounding: the chunk is taken another way)."""
    B, L, H, dk, dv = 1, 300, 2, 24, 40
    first, second, third = 0, 110, 150
    q, k, v, g, dy, state, dstate = make(6, B, L, H, 1, dk, dv, dtype)
    for t in (second, third):
        g[:, t] = -float("inf")
    for name in ("k", "v", "q", "dy", "g"):
        at = 131  # inside the chunk that the documents' border cuts
        args = dict(q=q.clone(), k=k.clone(), v=v.clone(), g=g.clone(), dy=dy.clone())
        x = args[name]
        x[0, at, 1] = bad if name == "g" else x[0, at, 1].index_fill(0, torch.tensor([3], device="cuda"), bad)
        clean = [wide(t) for t in (q, k, v, g)]
        ry, rs = block_ref.la(*clean, 1, 1.0, wide(state))
        sizes = [abs(t) for t in clean[:3]] + clean[3:]
        ay, as_ = block_ref.la(*sizes, 1, 1.0, abs(wide(state)))
        y, s, marks = hy.hyena_la_fwd_carry(args["q"], args["k"], args["v"], args["g"], state_in=state, want_marks=True)
        reach = slice(at, at + 1) if name == "q" else slice(at, third)
        touched = np.zeros(ry.shape, dtype=bool)
        if name != "dy":
            touched[:, reach, 1] = True
        close(y, np.where(touched, np.nan, ry), ay, dtype, name)
        close(s, rs, as_, "f32", name)
        if name != "dy":
            assert not torch.isfinite(y[0, at, 1]).all(), name
        dq, dk_, dv_, dg, dstate_in = hy.hyena_la_bwd(args["dy"], args["q"], args["k"], args["v"], args["g"], marks=marks, dstate_out=dstate,
                                                      want_dstate=True)
        ref = block_ref.la_grads(wide(dy), *clean, 1, 1.0, wide(state), wide(dstate))
        size = block_ref.la_grads(abs(wide(dy)), *sizes, 1, 1.0, abs(wide(state)), abs(wide(dstate)))
        # backwards, the second document alone may know of it: its other gradients at the other head and the other documents do not
        for what, gx, r, z in zip(("dq", "dk", "dv", "dg"), (dq, dk_, dv_, dg), ref, size):
            inside = np.zeros(r.shape, dtype=bool)
            inside[:, second:third, 1] = True
            close(gx, np.where(inside, np.nan, r), z, dtype, name + " " + what, extra=2e-5 * z.max() if what == "dg" else 0.0)
        close(dstate_in, ref[4], size[4], "f32", name + " dstate")
        # and of steps that come before, none of what only looks back
        if name in ("k", "v"):
            close(dq[:, second:at], ref[0][:, second:at], size[0][:, second:at], dtype, name + " dq before")
        if name in ("q", "dy"):
            close(dk_[:, at + 1:], ref[1][:, at + 1:], size[1][:, at + 1:], dtype, name + " dk behind")
            close(dv_[:, at + 1:], ref[2][:, at + 1:], size[2][:, at + 1:], dtype, name + " dv behind")


def within_range(q, k, v, g, dy, state, dstate, scale, dtype):
    """``check`` of whatever fp32 can hold: three factors of 2^50 are 2^150, so where the sum of the terms' magnitudes is 2^127 or more
    the sum may pass through an infinity on its way, whatever it is in the end."""
    group = v.shape[2] // q.shape[2]
    w = [wide(x) for x in (q, k, v, g)]
    a = [abs(x) for x in w[:3]] + w[3:]
    ref = block_ref.la(*w, group, scale, wide(state)) + block_ref.la_grads(wide(dy), *w, group, scale, wide(state), wide(dstate))
    size = (block_ref.la(*a, group, scale, abs(wide(state)))
            + block_ref.la_grads(abs(wide(dy)), *a, group, scale, abs(wide(state)), abs(wide(dstate))))
    y, s, marks = hy.hyena_la_fwd_carry(q, k, v, g, scale, state_in=state, want_marks=True)
    for given in (marks, None):
        got = (y, s) + hy.hyena_la_bwd(dy, q, k, v, g, scale, marks=given, state_in=state, dstate_out=dstate, want_dstate=True)
        for name, x, r, z in zip(("y", "state", "dq", "dk", "dv", "dg", "dstate"), got, ref, size):
            held = z < 2.0 ** 127
            assert held.mean() > 0.9, name
            extra = 2e-5 * z[held].max() if name == "dg" else 0.0
            close(x, np.where(held, r, np.nan), np.where(held, z, 0.0), "f32" if name in ("state", "dstate") else dtype, name, extra=extra)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,H,group,dk,dv", [(1, 200, 2, 2, 128, 200), (2, 130, 3, 1, 100, 64), (1, 70, 2, 1, 64, 128), (1, 65, 1, 1, 20, 33)])
def test_chunks_that_are_taken_a_step_at_a_time(B, L, H, group, dk, dv, dtype):
    """Numbers of 2^50 in one step: products of them are taken by the formulas, not at once, in every width, with shared heads and
    several tiles of columns, beside chunks that are; a scale that is not below one."""
    q, k, v, g, dy, state, dstate = make(12, B, L, H, group, dk, dv, dtype, resets=0.02)
    t = 40
    for x in (q, k, v, dy):
        x[:, t] *= 2.0 ** 50
    g[:, t + 1] = -float("inf")
    within_range(q, k, v, g, dy, state, dstate, 0.5, dtype)
    q, k, v, g, dy, state, dstate = make(13, B, L, H, group, dk, dv, dtype)
    check(q, k, v, g, dy, state, dstate, 37.0, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_states_that_are_not_finite_end_at_a_reset(dtype):
    """An infinity in the state in front, and in the gradient of the state behind: what lies across a reset does not know of them."""
    B, L, H, dk, dv = 1, 200, 2, 40, 72
    q, k, v, g, dy, state, dstate = make(14, B, L, H, 1, dk, dv, dtype)
    first, second = 21, 150
    g[:, [first, second]] = -float("inf")
    w = [wide(x) for x in (q, k, v, g)]
    a = [abs(x) for x in w[:3]] + w[3:]
    ry, rs = block_ref.la(*w, 1, 0.3, wide(state))
    ay, as_ = block_ref.la(*a, 1, 0.3, abs(wide(state)))
    ref = block_ref.la_grads(wide(dy), *w, 1, 0.3, wide(state), wide(dstate))
    size = block_ref.la_grads(abs(wide(dy)), *a, 1, 0.3, abs(wide(state)), abs(wide(dstate)))
    bad_in, bad_out = state.clone(), dstate.clone()
    bad_in[:, :, 3, 5] = float("inf")
    bad_out[:, :, 7, 11] = float("inf")
    y, s, marks = hy.hyena_la_fwd_carry(q, k, v, g, 0.3, state_in=bad_in, want_marks=True)
    touched = np.zeros(ry.shape, dtype=bool)
    touched[:, :first, :, 5] = True
    close(y, np.where(touched, np.nan, ry), ay, dtype, "y")
    close(s, rs, as_, "f32", "state")
    assert not torch.isfinite(y[:, 0, :, 5]).any()
    dq, dk_, dv_, dg, ds = hy.hyena_la_bwd(dy, q, k, v, g, 0.3, marks=marks, dstate_out=bad_out, want_dstate=True)
    for what, got, r, z, lo, hi in (("dq", dq, ref[0], size[0], first, L), ("dk", dk_, ref[1], size[1], 0, second), ("dv", dv_, ref[2], size[2], 0, second),
                                    ("dg", dg, ref[3], size[3], first, second + 1)):
        close(got[:, lo:hi], r[:, lo:hi], z[:, lo:hi], dtype, what, extra=2e-5 * z.max() if what == "dg" else 0.0)
    close(ds, ref[4], size[4], "f32", "dstate")


@pytest.mark.parametrize("dtype,group,dk,dv", [("bf16", 1, 128, 128), ("bf16", 2, 40, 72), ("f32", 3, 33, 20)])
def test_stretches_and_single_tokens_continue_each_other(dtype, group, dk, dv):
    B, L, H = 2, 170, 2 * group
    q, k, v, g, _, state, _ = make(8, B, L, H, group, dk, dv, dtype)
    w = [wide(x) for x in (q, k, v, g)]
    ry, rs = block_ref.la(*w, group, 0.3, wide(state))
    ay, as_ = block_ref.la(*[abs(x) for x in w[:3]], w[3], group, 0.3, abs(wide(state)))
    ys, s = [], state
    for lo, hi in ((0, 1), (1, 66), (66, 66), (66, 150)):
        y, s, _ = hy.hyena_la_fwd_carry(*(x[:, lo:hi] for x in (q, k, v, g)), 0.3, state_in=s)
        ys.append(y)
    for t in range(150, L):
        before = s
        ys.append(hy.hyena_la_step(*(x[:, t].contiguous() for x in (q, k, v, g)), s, 0.3)[:, None])
        assert s is before
    close(torch.cat(ys, 1), ry, ay, dtype, "y")
    close(s, rs, as_, "f32", "state")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,group,dk,dv", [(1, 1, 1, 1, 1), (3, 4, 2, 40, 72), (2, 2, 1, 300, 37), (1, 600, 1, 16, 132), (2, 3, 3, 64, 128)])
def test_a_single_token(B, H, group, dk, dv, dtype):
    q, k, v, g, _, state, _ = make(9, B, 1, H, group, dk, dv, dtype, resets=0.2)
    s0 = state.clone()
    guard = torch.full((B * H * dv + 64,), 7.0, dtype=v.dtype, device="cuda")
    out = guard[:B * H * dv].view(B, H, dv)
    y = hy.hyena_la_step(q[:, 0].contiguous(), k[:, 0].contiguous(), v[:, 0].contiguous(), g[:, 0].contiguous(), state, 0.5, out=out)
    w = [wide(x) for x in (q, k, v, g)]
    ry, rs = block_ref.la(*w, group, 0.5, wide(s0))
    ay, as_ = block_ref.la(*[abs(x) for x in w[:3]], w[3], group, 0.5, abs(wide(s0)))
    close(y[:, None], ry, ay, dtype, "y", mixed=False)
    close(state, rs, as_, "f32", "state")
    assert (guard[B * H * dv:] == 7).all()


def test_a_single_token_that_resets_forgets_nan():
    q, k, v, g, _, state, _ = make(9, 1, 1, 2, 1, 16, 16, "bf16")
    state[0, 0] = float("nan")
    g[0, 0, 0] = -float("inf")
    y = hy.hyena_la_step(q[:, 0].contiguous(), k[:, 0].contiguous(), v[:, 0].contiguous(), g[:, 0].contiguous(), state)
    assert torch.isfinite(y).all() and torch.isfinite(state).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_shared_rows_and_odd_places(dtype):
    """q, k, v as parts of one projection, a [L, B, ...] tensor, one key for all heads (distance 0), a gate that is the same at every
    step, inputs that begin between 16 bytes."""
    B, L, H, dk, dv = 2, 140, 3, 32, 48
    q, k, v, g, dy, state, dstate = make(11, B, L, H, 1, dk, dv, dtype)
    scale = 0.25
    dense = hy.hyena_la_fwd_carry(q, k, v, g, scale, state_in=state)[0]
    fused = torch.cat([q.flatten(2), k.flatten(2), v.flatten(2)], 2)
    fq, fk, fv = (x.unflatten(2, (H, -1)) for x in fused.split([H * dk, H * dk, H * dv], 2))
    assert torch.equal(hy.hyena_la_fwd_carry(fq, fk, fv, g, scale, state_in=state)[0], dense)
    tv, tg = v.transpose(0, 1).contiguous().transpose(0, 1), g.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(hy.hyena_la_fwd_carry(q, k, tv, tg, scale, state_in=state)[0], dense)
    odd = torch.empty(q.numel() + 3, dtype=q.dtype, device="cuda")[3:].view(q.shape).copy_(q)
    assert torch.equal(hy.hyena_la_fwd_carry(odd, k, v, g, scale, state_in=state)[0], dense)
    grads = hy.hyena_la_bwd(dy, q, k, v, g, scale, state_in=state, dstate_out=dstate)
    tdy = dy.transpose(0, 1).contiguous().transpose(0, 1)
    for a, b in zip(grads[:4], hy.hyena_la_bwd(tdy, odd, fk, fv, tg, scale, state_in=state, dstate_out=dstate)):
        assert torch.equal(a, b)
    one, same = k[:, :, :1].expand(B, L, H, dk), g[:, :1].expand(B, L, H)
    check(q, one, v, same, dy, state, dstate, scale, dtype, marks_too=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_end_where_they_end_and_are_the_same_every_time(dtype):
    B, L, H, dk, dv = 1, 1100, 2, 64, 72
    q, k, v, g, dy, state, dstate = make(12, B, L, H, 1, dk, dv, dtype, resets=0.01)
    n = v.numel()
    guard = torch.full((n + 256,), 5.0, dtype=v.dtype, device="cuda")
    y0, s0, m0 = hy.hyena_la_fwd_carry(q, k, v, g, state_in=state, want_marks=True, out=guard[:n].view(v.shape))
    assert (guard[n:] == 5).all()
    g0 = hy.hyena_la_bwd(dy, q, k, v, g, marks=m0, dstate_out=dstate, want_dstate=True)
    for _ in range(3):
        y, s, m = hy.hyena_la_fwd_carry(q, k, v, g, state_in=state, want_marks=True)
        assert torch.equal(y, y0) and torch.equal(s, s0) and torch.equal(m, m0)
        for a, b in zip(hy.hyena_la_bwd(dy, q, k, v, g, marks=m, dstate_out=dstate, want_dstate=True), g0):
            assert torch.equal(a, b)


def test_gradients_are_differences_of_the_forward_call():
    """fp32, along a random direction of each input: central differences of <y, dy> + <state, dstate>, whose own rounding (1e-6 of a
    sum of some 1e4 terms over a step of 1e-2) bounds the comparison."""
    q, k, v, g, dy, state, dstate = make(13, 1, 150, 2, 1, 16, 24, "f32")
    grads = hy.hyena_la_bwd(dy, q, k, v, g, 0.5, state_in=state, dstate_out=dstate, want_dstate=True)
    args = [q, k, v, g, state]

    def loss(a):
        y, s, _ = hy.hyena_la_fwd_carry(*a[:4], 0.5, state_in=a[4])
        return float((y.double() * dy).sum() + (s.double() * dstate).sum())

    rng = torch.Generator(device="cuda").manual_seed(1)
    for i, d in enumerate(grads):
        way = torch.randn(args[i].shape, generator=rng, device="cuda")
        if i == 3:
            way *= 0.1 * g.abs()
        up, down = (loss([a + s * 1e-2 * way if j == i else a for j, a in enumerate(args)]) for s in (1, -1))
        want = float((d.double() * way).sum())
        assert abs((up - down) / 2e-2 - want) <= 5e-3 * float((d.double() * way).abs().sum()) ** 0.5 + 2e-3 * abs(want) + 0.05, i


def test_empty_sequences_hand_their_states_on():
    q, k, v, g, dy, state, dstate = make(14, 2, 0, 2, 1, 8, 8, "bf16")
    y, s, _ = hy.hyena_la_fwd_carry(q, k, v, g, state_in=state)
    assert y.shape == v.shape and torch.equal(s, state)
    assert torch.equal(hy.hyena_la_fwd_carry(q, k, v, g)[1], torch.zeros_like(state))
    assert torch.equal(hy.hyena_la_bwd(dy, q, k, v, g, dstate_out=dstate, want_dstate=True)[4], dstate)


def test_refusals():
    q, k, v, g, dy, state, dstate = make(15, 1, 20, 2, 1, 16, 16, "bf16")
    for bad in (dict(k=k.float()), dict(k=k[:, :, :1]), dict(q=q[..., :8]), dict(g=g[..., :1]), dict(v=v.transpose(2, 3)), dict(q=q.cpu()),
                dict(state_in=state[:, :1]), dict(state_in=state.bfloat16())):
        with pytest.raises(ValueError):
            hy.hyena_la_fwd_carry(**{**dict(q=q, k=k, v=v, g=g), **bad})
    with pytest.raises(ValueError):
        hy.hyena_la_bwd(dy[:, :10], q, k, v, g)
    with pytest.raises(ValueError):
        hy.hyena_la_bwd(dy, q, k, v, g, marks=torch.empty(7, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        hy.hyena_la_step(q[:, 0].contiguous(), k[:, 0].contiguous(), v[:, 0].contiguous(), g[:, 0].contiguous(), None)
    with pytest.raises(TypeError):
        hy.hyena_la_fwd(q.half(), k.half(), v.half(), g.half())
    wide_k = torch.zeros(1, 4, 1, 129, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(hy.HyenaError):
        hy.hyena_la_fwd(wide_k, wide_k, v[:, :4], g[:, :4])
    with pytest.raises(ValueError):
        hy.hyena_la_fwd(q, k, torch.cat([v, v[:, :, :1]], 2), torch.cat([g, g[..., :1]], 2))   # 3 heads over 2
