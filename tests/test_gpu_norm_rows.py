"""Gradients of the norm over more rows than there are shares of dw, of rows that do not fit registers: the shares grow row after row."""
import numpy as np
import pytest

import block_ref
import paper_2503_01868_amd as hy
import test_gpu_norm as norm

from gpu_util import say

pytestmark = norm.pytestmark


@pytest.mark.parametrize("N,D,dtype", [(1100, 2050, "f32"), (1100, 8200, "f32"), (1100, 5003, "bf16"), (1500, 16400, "bf16")])
def test_shares_of_many_rows(N, D, dtype):
    say("norm bwd N=%d D=%d %s" % (N, D, dtype))
    dy, h, dh, w = norm.make(1, (N, D), dtype), norm.make(2, (N, D), dtype, 2.0), norm.make(3, (N, D), dtype), norm.make(4, (D,), dtype)
    rstd = hy.hyena_rmsnorm_fwd(h, w, eps=1e-5, want_rstd=True)[2]
    dx, dw = hy.hyena_rmsnorm_bwd(dy, h, rstd, w, dtotal=dh)
    rx, rw = block_ref.rmsnorm_grads(norm.wide(dy), norm.wide(h), norm.wide(w), norm.wide(dh), eps=1e-5)
    rr = 1 / np.sqrt((norm.wide(h) ** 2).mean(1, keepdims=True) + 1e-5)
    wdy = np.abs(norm.wide(dy) * norm.wide(w))
    norm.close(dx, rx, rr * (wdy + np.abs(norm.wide(h)) * rr ** 2 * (wdy * np.abs(norm.wide(h))).mean(1, keepdims=True)) + np.abs(norm.wide(dh)), dtype, "dx")
    norm.close(dw, rw, (np.abs(norm.wide(dy) * norm.wide(h)) * rr).sum(0), dtype, "dw")
