"""Host-only checks of the sizes that the entry points around the mixers refuse: what HIP cannot launch (2^32 threads and more)
is refused as unsupported before anything is enqueued."""
import ctypes

import pytest

from paper_2503_01868_amd import binding

UNSUPPORTED = 5
P = [ctypes.c_void_p(i << 46) for i in range(1, 17)]  # far apart, aligned, never looked at
LOTS = 1 << 45


def fwd(B, L, D, group=1, dtype=1, strides=None):
    return binding.lib().hyena_glr_fwd(*P[:4], None, P[4], None, None, strides, P[5], LOTS, B, L, D, group, dtype, None)


def bwd(B, L, D, group=1, dtype=1, marks=P[5]):
    return binding.lib().hyena_glr_bwd(*P[:5], marks, None, None, *P[6:10], None, None, P[10], LOTS, B, L, D, group, dtype, None)


@pytest.mark.parametrize("B,L,D,group", [(1, 1 << 30, 1, 1), (1, 64 * (1 << 23), 64, 64), (1 << 23, 1, 16, 1), (1 << 20, 512, 60, 1),
                                         (3, 1 << 32, 2, 1), (1, 1 << 29, 60, 3)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_recurrence_of_too_many_tiles(B, L, D, group, dtype):
    assert fwd(B, L, D, group, dtype) == UNSUPPORTED
    assert bwd(B, L, D, group, dtype) == UNSUPPORTED and bwd(B, L, D, group, dtype, marks=None) == UNSUPPORTED


def test_a_step_of_too_many_states():
    def step(B, D):
        return binding.lib().hyena_glr_step(*P[:6], B, D, 1, 1, None)

    assert step(1 << 32, 1) == UNSUPPORTED and step(1 << 20, 1 << 20) == UNSUPPORTED


@pytest.mark.parametrize("dtype", [0, 1])
def test_cross_entropy_of_too_many_tiles(dtype):
    lb = binding.lib()

    def xent_fwd(N, V, D):
        return lb.hyena_xent_fwd(*P[:5], P[5], LOTS, N, V, D, dtype, None)

    def xent_bwd(N, V, D):
        return lb.hyena_xent_bwd(*P[:7], P[7], LOTS, N, V, D, dtype, None)

    for call in (xent_fwd, xent_bwd):
        assert call(1 << 23, 10, 64) == UNSUPPORTED and call(10, 10, 1 << 23) == UNSUPPORTED
    # products of 2^38 elements: 2^24 tiles of 128 x 128
    assert xent_bwd(1 << 20, 100, 1 << 18) == UNSUPPORTED and xent_bwd(100, 1 << 20, 1 << 18) == UNSUPPORTED


def test_adamw_of_too_many_chunks():
    class Tensor(ctypes.Structure):
        _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "exp_avg", "exp_avg_sq", "avg_scale", "sq_scale", "master")] + [
            ("count", ctypes.c_int64), ("weight_decay", ctypes.c_float)]

    rows = (Tensor * 1)(Tensor(*(p.value for p in P[:4]), None, None, None, 4096 << 24, 0.0))
    assert binding.lib().hyena_adamw_table_bytes(rows, 1) == -1
    rows[0].count = 4096 * ((1 << 24) - 1)
    assert binding.lib().hyena_adamw_table_bytes(rows, 1) > 0
    assert binding.lib().hyena_adamw_step(P[0], 1, 1 << 24, 0, 0, 32, 0, 1e-3, 0.9, 0.95, 1e-8, 1, None, None) == 2
