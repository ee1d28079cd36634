"""Cross entropy over a vocabulary against its 64-bit form: sizes around the tiles and off every alignment, ignored rows, both
types, vocabularies taken in several pieces."""
import numpy as np
import pytest
import torch

import model_ref
import paper_2503_01868_amd as hy
from paper_2503_01868_amd import binding

from gpu_util import say

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def wide(t):
    return t.double().cpu().numpy()


def make(seed, N, V, D, dtype, ignored=0.2):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.normal(size=(N, D)).astype(np.float32)).to(DTYPES[dtype]).cuda()
    w = torch.from_numpy((rng.normal(size=(V, D)) * 2 / np.sqrt(D)).astype(np.float32)).to(DTYPES[dtype]).cuda()
    target = rng.integers(0, V, size=N)
    out = rng.uniform(size=N) < ignored
    target[out] = rng.choice([-100, -1, V, 1 << 40], size=out.sum())
    dloss = torch.from_numpy(rng.uniform(0.5, 1.5, size=N).astype(np.float32) / N).cuda()
    return x, w, torch.from_numpy(target).cuda(), dloss


def check(x, w, target, dloss, dtype):
    D = x.shape[1]
    X, W, T, d = wide(x), wide(w), target.cpu().numpy(), wide(dloss)
    loss, lse = hy.hyena_xent_fwd(x, w, target)
    rl, rs, z = model_ref.xent(X, W, T)
    # fp32 sums of D products: 4 sqrt(D) roundings of 2^-24 of the sum of magnitudes; exp, log and the sum over V: 2^-20
    dz = 4 * np.sqrt(D) * 2.0 ** -24 * (np.abs(X) @ np.abs(W).T).max()
    assert np.abs(wide(lse) - rs).max() <= dz + 2.0 ** -20 * (1 + np.abs(rs).max())
    assert np.abs(wide(loss) - rl).max() <= 2 * dz + 2.0 ** -20 * (1 + np.abs(rs).max())
    counts = (T >= 0) & (T < len(W))
    assert (loss[torch.from_numpy(~counts).cuda()] == 0).all()
    dx, dw = hy.hyena_xent_bwd(dloss, x, w, target, lse)
    rx, rw = model_ref.xent_grads(d, X, W, T)
    # an element of P is off by its parts times the logits' error, and by its own rounding where it becomes bf16
    p = np.exp(z - rs[:, None])
    p[np.flatnonzero(counts), T[counts]] += 1
    p *= np.where(counts, d, 0.0)[:, None]
    off = 2 * dz + 2.0 ** -20 + 4 * np.sqrt(max(x.shape[0], len(W))) * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    end = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    for name, got, ref, bound in (("dx", dx, rx, off * (p @ np.abs(W))), ("dw", dw, rw, off * (p.T @ np.abs(X)))):
        got = wide(got)
        assert np.isfinite(got).all()
        worst = (np.abs(got - ref) - (bound + end * np.abs(ref) + 1e-30)).max()
        assert worst <= 0, (name, worst)
    assert (dx[torch.from_numpy(~counts).cuda()] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,D", [(1, 1, 1), (1, 2, 8), (3, 5, 7), (64, 256, 64), (65, 257, 65), (128, 1000, 128), (130, 300, 72),
                                   (1, 5000, 256), (8, 777, 512), (17, 1000, 192), (33, 130, 64), (257, 129, 320), (300, 1030, 1000), (7, 70, 2048), (16, 1000, 40), (20, 333, 100), (64, 4097, 136), (48, 100, 4), (200, 300, 8), (129, 257, 1096),
                                   (4096, 3100, 64)])
def test_losses_and_gradients(N, V, D, dtype):
    say("xent N=%d V=%d D=%d %s" % (N, V, D, dtype))
    check(*make(N + V, N, V, D, dtype), dtype)


def test_a_vocabulary_in_pieces():
    N, V, D = 65600, 2500, 64
    say("xent in pieces N=%d V=%d D=%d" % (N, V, D))
    check(*make(2, N, V, D, "bf16"), "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_row_takes_part(dtype):
    x, w, target, dloss = make(3, 40, 100, 64, dtype, ignored=1.0)
    loss, lse = hy.hyena_xent_fwd(x, w, target)
    dx, dw = hy.hyena_xent_bwd(dloss, x, w, target, lse)
    assert (loss == 0).all() and torch.isfinite(lse).all() and (dx == 0).all() and (dw == 0).all()


def test_no_rows():
    w = torch.randn(10, 8, device="cuda")
    x, t = torch.empty(0, 8, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = hy.hyena_xent_fwd(x, w, t)
    dx, dw = hy.hyena_xent_bwd(loss, x, w, t, lse)
    assert loss.shape == (0,) and dx.shape == (0, 8) and (dw == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [5, 200])
def test_what_is_not_finite_in_a_row_that_takes_no_part_stays_out(N, dtype):
    x, w, target, dloss = make(4, N, 300, 128, dtype, ignored=0.0)
    target[2] = -100
    lse = hy.hyena_xent_fwd(x, w, target)[1]
    want = hy.hyena_xent_bwd(dloss, x, w, target, lse)
    x[2, 3], x[2, 4] = float("nan"), float("inf")
    loss, lse = hy.hyena_xent_fwd(x, w, target)
    got = hy.hyena_xent_bwd(dloss, x, w, target, lse)
    assert torch.isfinite(loss).all()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    target[2] = 1
    assert torch.isnan(hy.hyena_xent_fwd(x, w, target)[0][2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_logits(dtype):
    """Logits far beyond the exponential's range, equal ones, and one that takes the whole of its row."""
    x = torch.tensor([[300.0], [-300.0], [0.0]], device="cuda").to(DTYPES[dtype]).repeat(1, 64)
    w = torch.linspace(-1, 1, 5, device="cuda").to(DTYPES[dtype])[:, None].repeat(1, 64)
    target = torch.tensor([4, 4, 0], device="cuda")
    check(x, w, target, torch.ones(3, device="cuda"), dtype)


def test_fp32_values_at_the_ends_of_their_range():
    x = torch.full((2, 64), 3e38, device="cuda")
    w = torch.full((3, 64), 1e-38, device="cuda")
    loss, lse = hy.hyena_xent_fwd(x, w, torch.tensor([0, 2], device="cuda"))
    # every logit is 192; parts of w below fp32's normal numbers may be lost (2^-126 / 1e-38 of it)
    assert torch.isfinite(loss).all() and (loss - np.log(3)).abs().max() <= 1e-3 and (lse - 192 - np.log(3)).abs().max() <= 3


def test_the_same_every_time_and_inside_a_graph():
    x, w, target, dloss = make(5, 500, 3000, 256, "bf16")

    def step():
        loss, lse = hy.hyena_xent_fwd(x, w, target)
        return (loss, lse) + hy.hyena_xent_bwd(dloss, x, w, target, lse)

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        step()
    st.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(4):
        x.copy_(torch.randn_like(x))
        eager = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)


def test_on_another_stream_with_a_workspace_of_the_caller():
    x, w, target, dloss = make(6, 100, 500, 64, "bf16")
    want = hy.hyena_xent_fwd(x, w, target)
    need = binding.lib().hyena_xent_fwd_workspace_bytes(100, 500, 64, 1)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = hy.hyena_xent_fwd(x, w, target, workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(hy.HyenaError):
        hy.hyena_xent_fwd(x, w, target, workspace=ws[:need - 1])


def test_refusals():
    x, w, target, dloss = make(7, 10, 20, 64, "bf16")
    lse = torch.zeros(10, device="cuda")
    for bad in ((x.float(), w, target), (x, w[:, :32], target), (x, w, target.int()), (x, w, target[:5]), (x.cpu(), w, target),
                (x.t(), w, target), (x[:, ::2], w[:, ::2], target)):
        with pytest.raises(ValueError):
            hy.hyena_xent_fwd(*bad)
    with pytest.raises(TypeError):
        hy.hyena_xent_fwd(x.half(), w.half(), target)
    with pytest.raises(ValueError):
        hy.hyena_xent_bwd(dloss.double(), x, w, target, lse)
    with pytest.raises(ValueError):
        hy.hyena_xent_bwd(dloss, x, w, target, lse[:3])


@pytest.mark.parametrize("N,V,D", [(260, 11008, 36), (400, 390, 8300), (33, 40, 70), (64, 1000, 130), (1000, 50, 200), (7, 9000, 132)])
def test_float_rows_by_every_tile(N, V, D):
    """Tiles that are wider than high in either kind of product, tiles of few rows or short k, k divided among workgroups."""
    say("xent f32 %d x %d x %d" % (N, V, D))
    check(*make(N + V + D, N, V, D, "f32"), "f32")


def test_columns_that_begin_between_16_bytes():
    """The targets of a text are the text one further."""
    x, w, target, dloss = make(5, 101, 300, 64, "bf16")
    text, weights = (torch.cat([t[:1], t]) for t in (target, dloss))
    loss, lse = hy.hyena_xent_fwd(x, w, target)
    shifted = hy.hyena_xent_fwd(x, w, text[1:])
    assert torch.equal(loss, shifted[0]) and torch.equal(lse, shifted[1])
    column = torch.cat([lse[:1], lse])[1:]
    for a, b in zip(hy.hyena_xent_bwd(dloss, x, w, target, lse), hy.hyena_xent_bwd(weights[1:], x, w, text[1:], column)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("N,V,D", [(1, 100, 2), (100, 3000, 129), (128, 70, 264), (1024, 17000, 2048), (200, 33000, 1024)])
def test_few_bf16_rows(N, V, D):
    """The weights read as they lie, odd widths and vocabularies that end inside a step; the last two are few rows for their weights."""
    say("xent bf16 %d x %d x %d" % (N, V, D))
    if N * V <= 1 << 22:
        check(*make(N + V + D, N, V, D, "bf16"), "bf16")
        return
    # against the gradient of x alone: rows by the others' rules agree with the same rows in a call of more of them
    x, w, target, dloss = make(N + V + D, N, V, D, "bf16")
    loss, lse = hy.hyena_xent_fwd(x, w, target)
    dx, _ = hy.hyena_xent_bwd(dloss, x, w, target, lse)
    z = x.float() @ w.float().t()
    p = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
    counts = (target >= 0) & (target < V)
    p[counts, target[counts]] -= 1
    p *= torch.where(counts, dloss, 0.0)[:, None]
    ref, mass = p @ w.float(), p.abs() @ w.float().abs()
    # P's rounding to bf16 (2^-8 with its ends), the logits' in fp32, and the result's
    assert ((dx.float() - ref).abs() <= 2.0 ** -7 * mass + 2.0 ** -8 * ref.abs() + 1e-30).all()
