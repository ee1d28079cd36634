"""The norm, the linear attention, the loss and the choice of tokens as a model uses them together: a block's gradients against torch's own in
64 bits, training and writing inside graphs that are replayed between eager work, and two of them at once on two streams."""
import pytest
import torch

import paper_2503_01868_amd as hy

from gpu_util import say

pytestmark = pytest.mark.gpu

B, L, D, H, GROUP, DK, DV, V = 2, 70, 48, 4, 2, 24, 20, 40


def weights(dtype, device="cuda"):
    g = torch.Generator().manual_seed(1)

    def w(*shape):
        return (torch.randn(*shape, generator=g, dtype=torch.float64) * shape[-1] ** -0.5).to(device=device, dtype=dtype)

    return dict(n1=w(D) + 1, n2=w(D) + 1, wq=w(H // GROUP * DK, D), wk=w(H // GROUP * DK, D), wv=w(H * DV, D), wg=w(H, D), wo=w(D, H * DV), words=w(V, D))


def inputs(dtype, seed=2, device="cuda", rows=(B, L)):
    g = torch.Generator().manual_seed(seed)
    x, r = (torch.randn(*rows, D, generator=g, dtype=torch.float64).to(device=device, dtype=dtype) for _ in range(2))
    return x, r, torch.randint(0, V, (rows[0] * (rows[1] if len(rows) > 1 else 1),), generator=g).to(device)


def heads(y, w):
    """q, k, v and log decays of normed rows."""
    lead = y.shape[:-1]
    q, k = ((y @ w[n].t()).view(*lead, H // GROUP, DK) for n in ("wq", "wk"))
    return q, k, (y @ w["wv"].t()).view(*lead, H, DV), -torch.exp(y @ w["wg"].t() - 1)


def block(x, r, targets, w):
    """The loss of each token and the gradients of x and the norms' weights, with the package's calls."""
    y, total, rstd = hy.hyena_rmsnorm_fwd(x, w["n1"], residual=r, want_rstd=True)
    q, k, v, g = heads(y, w)
    a, _, marks = hy.hyena_la_fwd_carry(q, k, v, g, DK ** -0.5, want_state=False, want_marks=True)
    o = a.view(*x.shape[:-1], H * DV) @ w["wo"].t()
    y2, total2, rstd2 = hy.hyena_rmsnorm_fwd(o, w["n2"], residual=total, want_rstd=True)
    loss, lse = hy.hyena_xent_fwd(y2.view(-1, D), w["words"], targets)
    dy2, _ = hy.hyena_xent_bwd(torch.full_like(loss, 1.0), y2.view(-1, D), w["words"], targets, lse)
    do, dn2 = hy.hyena_rmsnorm_bwd(dy2.view(x.shape), total2, rstd2, w["n2"])
    da = (do @ w["wo"]).view(a.shape)
    dq, dk, dv, dg, _ = hy.hyena_la_bwd(da, q, k, v, g, DK ** -0.5, marks=marks)
    lead = x.shape[:-1]
    dy = dq.view(*lead, -1) @ w["wq"] + dk.view(*lead, -1) @ w["wk"] + dv.view(*lead, -1) @ w["wv"] + (dg * g) @ w["wg"]
    dx, dn1 = hy.hyena_rmsnorm_bwd(dy, total, rstd, w["n1"], dtotal=do)
    return loss, dx, dn1, dn2


def test_a_block_and_its_gradients():
    """fp32: a gradient passes some thousand roundings of 2^-24 in a row at most, 6e-5 of the largest; twice that for the two ways."""
    say("block")
    w, (x, r, targets) = weights(torch.float32), inputs(torch.float32)
    loss, dx, dn1, dn2 = block(x, r, targets, w)
    w64 = {n: t.double().cpu() for n, t in w.items()}
    x64, r64 = x.double().cpu().requires_grad_(), r.double().cpu()
    w64["n1"].requires_grad_(), w64["n2"].requires_grad_()

    def norm(h, n):
        return h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6) * n

    total = x64 + r64
    q, k, v, g = heads(norm(total, w64["n1"]), w64)
    q, k = (t.repeat_interleave(GROUP, 2) for t in (q, k))
    S, out = torch.zeros(B, H, DK, DV, dtype=torch.float64), []
    for t in range(L):
        S = torch.exp(g[:, t])[..., None, None] * S + k[:, t, :, :, None] * v[:, t, :, None, :]
        out.append(DK ** -0.5 * (q[:, t, :, :, None] * S).sum(2))
    o = torch.stack(out, 1).reshape(B, L, H * DV) @ w64["wo"].t()
    logits = (norm(o + total, w64["n2"]) @ w64["words"].t()).reshape(-1, V)
    ref = torch.nn.functional.cross_entropy(logits, targets.cpu(), reduction="none")
    ref.sum().backward()
    for name, got, want in (("loss", loss, ref.detach()), ("dx", dx, x64.grad), ("dn1", dn1, w64["n1"].grad), ("dn2", dn2, w64["n2"].grad)):
        assert (got.double().cpu() - want).abs().max() <= 1.2e-4 * want.abs().max(), name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_training_inside_a_graph(dtype):
    """Every replay gives the eager call's bits, with eager calls of the same sizes and synchronizations between them."""
    say("block graph %s" % dtype)
    w = weights(dtype)
    x, r, targets = inputs(dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(x, r, targets, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = block(x, r, targets, w)
    for seed in (2, 5, 6, 7):
        for at, new in zip((x, r, targets), inputs(dtype, seed)):
            at.copy_(new)
        graph.replay()
        got = [t.clone() for t in made]
        torch.cuda.synchronize()
        for a, b in zip(got, block(x, r, targets, w)):
            assert torch.equal(a, b), seed


def write(x, r, u, state, w):
    """One token of every sequence."""
    y, total, _ = hy.hyena_rmsnorm_fwd(x, w["n1"], residual=r)
    q, k, v, g = heads(y, w)
    o = hy.hyena_la_step(q, k, v, g, state, DK ** -0.5).view(-1, H * DV) @ w["wo"].t()
    y8, scale, total, _ = hy.hyena_rmsnorm_fwd_8bit(o, w["n2"], residual=total)
    logits = (y8.float() * scale[:, None]).to(x.dtype) @ w["words"].t()
    return hy.hyena_sample(logits, u, 0.8, 20, 0.95, 0.01) + (total,)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_writing_inside_a_graph(dtype):
    N = 5
    w = weights(dtype)
    x, r, _ = inputs(dtype, rows=(N,))
    u = torch.rand(N, device="cuda")
    state = torch.zeros(N, H, DK, DV, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        write(x, r, u, state, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        made = write(x, r, u, state, w)
    state.zero_()
    eager = state.clone()
    for seed in range(3, 9):
        new = inputs(dtype, seed, rows=(N,))
        x.copy_(new[0]), r.copy_(new[1]), u.copy_(torch.rand(N, device="cuda"))
        graph.replay()
        got = [t.clone() for t in made]
        torch.cuda.synchronize()
        for a, b in zip(got, write(x, r, u, eager, w)):
            assert torch.equal(a, b), seed
        assert torch.equal(state, eager)


def test_two_streams_at_once():
    """Each with workspaces of its own: neither disturbs the other."""
    w = weights(torch.bfloat16)
    sets = [inputs(torch.bfloat16, s) for s in (11, 12)]
    alone = [block(*s, w) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        made = []
        for s, args in zip(streams, sets):
            with torch.cuda.stream(s):
                made.append(block(*args, w))
        torch.cuda.synchronize()
        for got, want in zip(made, alone):
            assert all(torch.equal(a, b) for a, b in zip(got, want))
