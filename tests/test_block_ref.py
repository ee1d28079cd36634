"""The 64-bit forms of linear attention and the norm against differences and hand-made cases; the choice of tokens against counts."""
import math

import numpy as np
import pytest

import block_ref


def directional(f, args, grads, rng):
    """d f along a random direction by central differences and by the gradients."""
    for i, (x, d) in enumerate(zip(args, grads)):
        way = rng.normal(size=x.shape)
        way[~np.isfinite(x)] = 0.0
        h = 1e-5
        up, down = (f(*[a + s * h * way if j == i else a for j, a in enumerate(args)]) for s in (1, -1))
        assert abs((up - down) / (2 * h) - (d * way).sum()) <= 1e-6 * (1 + abs((d * way).sum())), i


@pytest.mark.parametrize("group,forget", [(1, False), (2, True), (3, True)])
def test_gradients_of_linear_attention_are_differences(group, forget):
    rng = np.random.default_rng(group)
    B, L, H, dk, dv = 2, 9, 2 * group, 3, 4
    q, k = rng.normal(size=(2, B, L, H // group, dk))
    v, dy = rng.normal(size=(2, B, L, H, dv))
    g = -np.exp(rng.normal(size=(B, L, H)))
    if forget:
        g[:, 4] = -np.inf
    state, dstate = rng.normal(size=(2, B, H, dk, dv))

    def loss(q, k, v, g, state):
        y, S = block_ref.la(q, k, v, g, group, 0.7, state)
        return (y * dy).sum() + (S * dstate).sum()

    directional(loss, (q, k, v, g, state), block_ref.la_grads(dy, q, k, v, g, group, 0.7, state, dstate), rng)


def test_linear_attention_without_decay_is_attention_without_softmax():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(3, 1, 7, 1, 5))
    p = np.tril(q[0, :, 0] @ k[0, :, 0].T)
    y, S = block_ref.la(q, k, v, np.zeros((1, 7, 1)))
    np.testing.assert_allclose(y[0, :, 0], p @ v[0, :, 0], rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(S[0, 0], k[0, :, 0].T @ v[0, :, 0], rtol=1e-12, atol=1e-12)


def test_a_decay_of_zero_forgets_what_is_not_finite():
    q, k, v = np.ones((3, 1, 4, 1, 1))
    v[0, 1] = np.nan
    g = np.zeros((1, 4, 1))
    g[0, 2] = -np.inf
    y, S = block_ref.la(q, k, v, g)
    assert y[0, 0, 0, 0] == 1 and math.isnan(y[0, 1, 0, 0]) and y[0, 2, 0, 0] == 1 and y[0, 3, 0, 0] == 2 and S[0, 0, 0, 0] == 2


@pytest.mark.parametrize("weights,along", [(True, True), (False, False)])
def test_gradients_of_the_norm_are_differences(weights, along):
    rng = np.random.default_rng(3)
    h, dy, dh = rng.normal(size=(3, 5, 6))
    w = rng.normal(size=6) if weights else None
    dx, dw = block_ref.rmsnorm_grads(dy, h, w, dh if along else None)

    def loss(h, w=None):
        y, total, _ = block_ref.rmsnorm(h, w)
        return (y * dy).sum() + ((total * dh).sum() if along else 0.0)

    directional(loss, (h, w) if weights else (h,), (dx, dw) if weights else (dx,), rng)


def test_tokens_by_hand():
    z = np.log([0.1, 0.4, 0.2, 0.3])
    assert [block_ref.sample(z, u)[0] for u in (0.0, 0.099, 0.101, 0.499, 0.501, 0.699, 0.701, 1.0)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [block_ref.sample(z, u, top_k=2)[0] for u in (0.0, 0.57, 0.58)] == [1, 1, 3]
    assert [block_ref.sample(z, u, top_p=0.71)[0] for u in (0.0, 0.44, 0.45, 0.66, 0.67)] == [1, 1, 2, 2, 3]
    assert [block_ref.sample(z, u, min_p=0.6)[0] for u in (0.0, 0.57, 0.58)] == [1, 1, 3]
    assert block_ref.sample(z, 0.9, temperature=0) == (1, 1.0)
    assert block_ref.sample([2.0, 2.0, 1.0, 2.0], 0.99, top_k=2)[0] == 1       # the lowest of equal ones
    assert block_ref.sample([-math.inf] * 3, 0.5) == (-1, 0.0)
    assert block_ref.sample([0.0, math.inf, math.inf], 0.6)[0] == 2


def test_tokens_come_as_often_as_they_are_likely():
    z = np.array([0.0, 1.0, -1.0, 2.0])
    p = np.exp(z / 0.8) / np.exp(z / 0.8).sum()
    got = [block_ref.sample(z, (i + 0.5) / 1000, 0.8) for i in range(1000)]
    counts = np.bincount([t for t, _ in got], minlength=4) / 1000
    assert np.abs(counts - p).max() <= 1e-3
    assert all(abs(prob - p[t]) < 1e-12 for t, prob in got)
