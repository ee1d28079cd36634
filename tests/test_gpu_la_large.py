"""The single token of the linear attention over states that are read as a stream (64 MiB and more)."""
import pytest
import torch

import paper_2503_01868_amd as hy

from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,group,dk,dv", [(32, 32, 1, 128, 128), (33, 20, 2, 100, 260)])
def test_a_single_token_over_large_states(B, H, group, dk, dv):
    """Against torch's double.  The decay is the square of a power of two whose last bit may be off, 2 x 2^-23, of an argument of at most
    0.73 that is rounded to 2^-25, 2 x 0.7 x 2^-25; it is multiplied in twice, 2 x 2^-24; the product of k and v and the sum round
    once each, 2 x 2^-24: together below 2^-22 + 2^-24 + 2^-23 + 2^-23 < 2^-21 x 1.2 of the terms' magnitudes."""
    say("la step of large states B=%d" % B)
    gen = torch.Generator(device="cuda").manual_seed(B)
    q, k = (torch.randn(B, H // group, dk, generator=gen, device="cuda") for _ in range(2))
    v, g = torch.randn(B, H, dv, generator=gen, device="cuda"), -torch.rand(B, H, generator=gen, device="cuda")
    g[1, 2] = -float("inf")
    state = torch.randn(B, H, dk, dv, generator=gen, device="cuda")
    assert state.numel() * 4 >= 1 << 26
    kh, qh = (x.double().repeat_interleave(group, 1) for x in (k, q))
    kept = torch.exp(g.double())[..., None, None] * state.double()
    added = kh[..., :, None] * v.double()[..., None, :]
    want = kept + added
    y = hy.hyena_la_step(q, k, v, g, state, 0.3)
    assert ((state.double() - want).abs() <= 1.2 * 2.0 ** -21 * (kept.abs() + added.abs()) + 1e-30).all()
    ref = 0.3 * (qh[..., :, None] * want).sum(2)
    size = 0.3 * (qh.abs()[..., :, None] * (kept.abs() + added.abs())).sum(2)
    assert ((y.double() - ref).abs() <= 2e-5 * size).all()
