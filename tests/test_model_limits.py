"""Host-only checks of the sizes that the entry points around the mixers refuse: what HIP cannot launch (2^32 threads and more)
is refused as unsupported before anything is enqueued."""
import ctypes
import time

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


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_vocabulary_of_any_size_is_sized_at_once(dtype):
    """Two sizes of pieces occur, however many pieces there are: 2^49 words take no longer than 2^20."""
    lb = binding.lib()
    sizes = (lb.hyena_xent_fwd_workspace_bytes, lb.hyena_xent_bwd_workspace_bytes)
    for N, D in ((64, 8), (1000, 8), (8, 7), (1, 1)):
        begin = time.perf_counter()
        for size in sizes:
            assert size(N, 1 << 48, D, dtype) > 0
            size(N, (1 << 49) + 12345, D, dtype)
        assert time.perf_counter() - begin < 0.05
    for size in sizes:  # what cannot be launched has no size
        assert size(1 << 23, 10, 64, dtype) == -1 == size(10, 10, 1 << 23, dtype) and size(1 << 60, 1, 1, dtype) == -1
        assert size(1, 1, 1 << 60, dtype) == -1


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("N,V,D", [(64, 5000, 64), (65, 70000, 1000), (300, 33001, 999), (4000, 1 << 20, 512), (1 << 20, 1500, 64), (1 << 20, 2100, 72),
                                   (131072, 1024, 64), (131072, 1025, 64), (8192, 65536, 4096), (2, (1 << 23) + 5, 8)])
def test_the_workspace_holds_pairs_targets_and_copies(N, V, D, dtype):
    """Against sums piece by piece, written out here from what a call keeps: the pairs of a row's tiles, the targets' values and
    the copies of rows that do not begin where 16 bytes do."""
    lb = binding.lib()
    e, packed = 4 if dtype == 0 else 2, dtype == 1 and D % 8 != 0
    up = lambda n, to: -(-n // to) * to  # noqa: E731
    most = min(max(1024, (512 << 20) // (2 * e * up(N, 64)) // 256 * 256), 1 << 22)
    piece = min(up(-(-V // -(-V // most)), 256), up(V, 64))
    cols = [min(piece, V - v) for v in range(0, V, piece)]
    if dtype == 0 and N <= 32 and D % 4 == 0:
        tiles = -(-V // 64)
    else:
        tiles = sum(-(-c // (64 if N <= 64 else 128)) for c in cols)
    need = up(N * tiles * 8, 256) + up(N * 4, 256)
    if packed:
        need += up(N * up(D, 64) * 2, 256) + up(min(piece, V) * up(D, 64) * 2, 256)
    assert lb.hyena_xent_fwd_workspace_bytes(N, V, D, dtype) == need
