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
