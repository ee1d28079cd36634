"""Linear attention of no heads: nothing, if q and k have none either, and otherwise refused (rows of q that belong to no head would have
gradients that nobody writes)."""
import pytest
import torch

import paper_2503_01868_amd as hy

pytestmark = pytest.mark.gpu


def test_no_heads():
    q, v, g = torch.zeros(2, 5, 0, 8, device="cuda"), torch.zeros(2, 5, 0, 16, device="cuda"), torch.zeros(2, 5, 0, device="cuda")
    y, state, marks = hy.hyena_la_fwd_carry(q, q, v, g, want_marks=True)
    assert y.shape == v.shape and state.shape == (2, 0, 8, 16)
    dq, dk, dv, dg, dstate = hy.hyena_la_bwd(v, q, q, v, g, marks=marks, want_dstate=True)
    assert dq.shape == dk.shape == q.shape and dv.shape == v.shape and dg.shape == g.shape and dstate.shape == state.shape
    assert hy.hyena_la_step(q[:, 0], q[:, 0], v[:, 0], g[:, 0], state).shape == (2, 0, 16)
    two = torch.zeros(2, 5, 2, 8, device="cuda")
    with pytest.raises(ValueError):
        hy.hyena_la_fwd(two, two, v, g)
    with pytest.raises(ValueError):
        hy.hyena_la_bwd(v, two, two, v, g)
    with pytest.raises(ValueError):
        hy.hyena_la_step(two[:, 0].contiguous(), two[:, 0].contiguous(), v[:, 0], g[:, 0], state)
    with pytest.raises(ValueError):
        hy.hyena_la_fwd(q, q, torch.zeros(2, 5, 3, 16, device="cuda"), torch.zeros(2, 5, 3, device="cuda"))
