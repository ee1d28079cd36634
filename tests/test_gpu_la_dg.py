"""Gradients of the log decays where they are nothing, or little beside what a step says to itself."""
import numpy as np
import pytest
import torch

import block_ref
import paper_2503_01868_amd as hy
import test_gpu_la as la

from gpu_util import say

pytestmark = la.pytestmark


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,group,dk,dv", [(4, 2, 2, 128, 64), (2, 3, 1, 40, 130), (7, 4, 1, 16, 16)])
def test_a_first_step_without_a_state_has_none(B, H, group, dk, dv, dtype):
    """There is nothing in front of its decay."""
    say("la dg of one step B=%d H=%d dk=%d dv=%d %s" % (B, H, dk, dv, dtype))
    q, k, v, g, dy, _, dstate = la.make(1, B, 1, H, group, dk, dv, dtype)
    for behind in (None, dstate):
        assert (hy.hyena_la_bwd(dy, q, k, v, g, 0.3, dstate_out=behind)[3] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("decay", [-8.0, -20.0, -60.0])
def test_strong_decays(decay, dtype):
    """dg is e^decay of what a step says to itself.  It is a difference of sums over pairs of steps of a chunk: each pair that reaches over any
    decay is a term of the gradient of one of them, so that the error is 2e-5 of all the chunk's gradients' terms; bf16: a term passes a rounding,
    and the stored element another."""
    say("la dg strong decays %g %s" % (decay, dtype))
    q, k, v, g, dy, state, dstate = la.make(2, 2, 150, 2, 1, 48, 72, dtype)
    g.fill_(decay)
    w = [la.wide(x) for x in (q, k, v, g)]
    a = [abs(x) for x in w[:3]] + w[3:]
    ref = block_ref.la_grads(la.wide(dy), *w, 1, 0.3, la.wide(state), la.wide(dstate))[3]
    size = block_ref.la_grads(abs(la.wide(dy)), *a, 1, 0.3, abs(la.wide(state)), abs(la.wide(dstate)))[3]
    got = la.wide(hy.hyena_la_bwd(dy, q, k, v, g, 0.3, state_in=state, dstate_out=dstate)[3])
    chunk = np.concatenate([np.broadcast_to(c.sum(1, keepdims=True), c.shape) for c in np.split(size, range(64, 150, 64), 1)], 1)
    bound = 2e-5 * chunk + (2.0 ** -8 * size + 2.0 ** -8 * abs(ref) if dtype == "bf16" else 0.0)
    assert (abs(got - ref) <= bound).all(), (abs(got - ref) / bound).max()
