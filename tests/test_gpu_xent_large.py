"""Cross entropy at sizes where tiles, pieces of the vocabulary and launches change: against the 64-bit form."""
import numpy as np
import pytest
import torch

import model_ref
import paper_2503_01868_amd as hy

from gpu_util import say

pytestmark = pytest.mark.gpu


def test_rows_that_are_copied_and_have_more_than_2_to_the_32_numbers():
    """A width of 4097 is copied to rows of 4160, a number a lane: more than HIP launches threads.  Rows of the beginning, of the
    end and around the 2^32nd number, against the 64-bit form: 4 sqrt(D) roundings of 2^-24 of the sum of magnitudes for the
    logits, 2^-20 for the exponentials and their sum."""
    N, V, D = (1 << 32) // 4160 + 300, 50, 4097
    say("xent rows of %d numbers" % (N * D))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    x = torch.empty(N, D, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    w = torch.empty(V, D, dtype=torch.bfloat16, device="cuda").normal_(std=2 / np.sqrt(D), generator=gen)
    target = torch.randint(0, V, (N,), generator=gen, device="cuda")
    loss, lse = hy.hyena_xent_fwd(x, w, target)
    W = w.double().cpu().numpy()
    for at in (0, (1 << 32) // 4160 - 50, N - 100):
        X, T = x[at:at + 100].double().cpu().numpy(), target[at:at + 100].cpu().numpy()
        rl, rs, _ = model_ref.xent(X, W, T)
        dz = 4 * np.sqrt(D) * 2.0 ** -24 * (np.abs(X) @ np.abs(W).T).max()
        end = 2.0 ** -20 * (1 + np.abs(rs).max())
        assert np.abs(lse[at:at + 100].double().cpu().numpy() - rs).max() <= dz + end
        assert np.abs(loss[at:at + 100].double().cpu().numpy() - rl).max() <= 2 * dz + end


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V,at", [(3, 5, 2), (200, 300, 290), (40, 300, 3)])
def test_losses_that_are_small_beside_their_logits(N, V, at, dtype):
    """A target at 40, four words at 25, the others at -40: the loss is log(1 + 4 e^-15), 1.2e-6, where numbers of 40 are 3.8e-6
    apart.  Four additions to 1, the logarithm and the joins of tiles: 8 roundings of 2^-24 at the most.  (All products are exact.)"""
    x = torch.ones(N, 64, device="cuda", dtype=dtype)
    w = torch.full((V, 64), -0.625, device="cuda", dtype=dtype)
    w[at] = 0.625
    w[[(at + i) % V for i in range(1, 5)]] = 0.390625
    loss, lse = hy.hyena_xent_fwd(x, w, torch.full((N,), at, device="cuda"))
    assert (lse == 40).all()
    assert (loss.double() - np.log1p(4 * np.exp(-15.0))).abs().max() <= 8 * 2.0 ** -24


DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(seed, N, V, D, dtype, ignored=0.2):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(N, D, generator=gen, device="cuda").to(DTYPES[dtype])
    w = (torch.randn(V, D, generator=gen, device="cuda") * 2 / np.sqrt(D)).to(DTYPES[dtype])
    target = torch.randint(0, V, (N,), generator=gen, device="cuda")
    out = torch.rand(N, generator=gen, device="cuda") < ignored
    target = torch.where(out, torch.tensor([-100, -1, V, 1 << 40], device="cuda")[target % 4], target)
    dloss = (0.5 + torch.rand(N, generator=gen, device="cuda")) / N
    return x, w, target, dloss


def check(x, w, target, dloss, dtype):
    """Losses and gradients against their definition in 64 bits.  A logit is a fp32 sum of D products: 4 sqrt(D) roundings of 2^-24
    of the sum of magnitudes; exp, log and the sum over V: 2^-20.  An element of P is off by its parts times the logits' error,
    and by its own rounding where it becomes bf16; its products by 4 sqrt(k) roundings and the result's own."""
    D, V = x.shape[1], w.shape[0]
    X, W, d = x.double(), w.double(), dloss.double()
    z = X @ W.t().contiguous()
    rs = torch.logsumexp(z, 1)
    counts = (target >= 0) & (target < V)
    rows = torch.nonzero(counts)[:, 0]
    rl = torch.zeros_like(rs)
    rl[rows] = rs[rows] - z[rows, target[rows]]
    dz = float(4 * np.sqrt(D) * 2.0 ** -24 * (X.abs() @ W.abs().t().contiguous()).max())
    end = float(2.0 ** -20 * (1 + rs.abs().max()))
    loss, lse = hy.hyena_xent_fwd(x, w, target)
    assert (lse.double() - rs).abs().max() <= dz + end
    assert (loss.double() - rl).abs().max() <= 2 * dz + end and (loss[~counts] == 0).all()
    dx, dw = hy.hyena_xent_bwd(dloss, x, w, target, lse)
    p = torch.exp(z - rs[:, None]) * torch.where(counts, d, 0.0)[:, None]
    del z
    one = torch.zeros_like(p)
    one[rows, target[rows]] = d[rows]
    off = 2 * dz + 2.0 ** -20 + 4 * np.sqrt(max(x.shape[0], V)) * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    own = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
    for name, got, ref, mass in (("dx", dx, (p - one) @ W, (p + one) @ W.abs()),
                                 ("dw", dw, (p - one).t().contiguous() @ X, (p + one).t().contiguous() @ X.abs())):
        assert torch.isfinite(got).all(), name
        worst = float(((got.double() - ref).abs() - (off * mass + own * ref.abs() + 1e-30)).max())
        assert worst <= 0, (name, worst)
    assert (dx[~counts] == 0).all()


@pytest.mark.parametrize("D", [40, 37])
def test_float_pieces_that_end_inside_a_tile(D):
    """Tiles of 192 columns over pieces of 2048: the first piece's last tile ends among the next one's targets."""
    N, V = 20481, 3900
    say("xent f32 in pieces %d x %d x %d" % (N, V, D))
    x, w, target, dloss = make(3, N, V, D, "f32")
    target[::3] = 2040 + torch.arange(len(target[::3]), device="cuda") % 160
    check(x, w, target, dloss, "f32")


@pytest.mark.parametrize("N,V,D", [(3553, 3601, 3592), (1024, 17000, 2048), (200, 33000, 1024), (4099, 8191, 4104)])
def test_tiles_of_256(N, V, D):
    """Logits, P in both orders and both products in tiles of 256 x 256, ragged in every direction (and calls of few rows for their
    weights, which take some of them)."""
    say("xent bf16 %d x %d x %d" % (N, V, D))
    check(*make(N + V + D, N, V, D, "bf16"), "bf16")


@pytest.mark.parametrize("N,V,D,dtype", [(65600, 2500, 65, "bf16"), (40, 2200000, 16, "bf16"), (40, 2200000, 9, "bf16"), (33, 1100000, 12, "f32"),
                                         (20, 1100000, 12, "f32"), (9000, 16000, 72, "bf16"), (16000, 9100, 520, "bf16")])
def test_vocabularies_in_pieces(N, V, D, dtype):
    """Rows that are copied, few rows against millions of words, and pieces of large tiles."""
    say("xent %s in pieces %d x %d x %d" % (dtype, N, V, D))
    check(*make(N + V + D, N, V, D, dtype), dtype)


def test_losses_alone_of_every_tile_agree_with_each_other():
    """The losses of some rows, in a call of them alone and among others: the same numbers but for the order of the sums over V."""
    x, w, target, _ = make(9, 2000, 6000, 512, "bf16", ignored=0.0)
    loss, lse = hy.hyena_xent_fwd(x, w, target)
    bound = 2.0 ** -20 * (1 + float(lse.abs().max())) + 8 * np.sqrt(512) * 2.0 ** -24 * float((x[:1].float().abs() @ w.float().abs().t()).max())
    for rows in (1, 30, 60, 100, 300):
        some = hy.hyena_xent_fwd(x[:rows], w, target[:rows])
        assert (some[0] - loss[:rows]).abs().max() <= bound and (some[1] - lse[:rows]).abs().max() <= bound
