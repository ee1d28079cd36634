"""The 64-bit forms that the GPU tests compare with: gradients against differences, and closed forms."""
import numpy as np
import pytest

import model_ref


def difference(f, x, h=1e-5):
    """Central differences of the scalar f in every element of x."""
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + h
        up = f()
        x[i] = keep - h
        d[i] = (up - f()) / (2 * h)
        x[i] = keep
    return d


@pytest.mark.parametrize("B,L,D,group", [(1, 1, 1, 1), (2, 5, 4, 2), (1, 7, 6, 3)])
def test_recurrence_gradients_match_differences(B, L, D, group):
    rng = np.random.default_rng(10 + L)
    q, k, v, dy = (rng.normal(size=(B, L, D)) for _ in range(4))
    g = -rng.uniform(0.01, 2, size=(B, L, D // group))
    state, dstate = rng.normal(size=(B, D)), rng.normal(size=(B, D))

    def loss():
        y, s, _ = model_ref.glr(q, k, v, g, group, state)
        return (y * dy).sum() + (s * dstate).sum()

    grads = model_ref.glr_grads(dy, q, k, v, g, group, state, dstate)
    for got, x in zip(grads, (q, k, v, g, state)):
        # central differences: h^2 / 6 times the third derivative, and 1e-16 / h from cancellation
        np.testing.assert_allclose(got, difference(loss, x), rtol=1e-6, atol=1e-7)


def test_recurrence_of_a_constant_decay_is_a_geometric_sum():
    L, decay = 40, 0.9
    one = np.ones((1, L, 1))
    y, s, _ = model_ref.glr(one, one, one, np.log(decay) * one)
    np.testing.assert_allclose(y[0, :, 0], (1 - decay ** np.arange(1, L + 1)) / (1 - decay), rtol=1e-12)
    assert s[0, 0] == y[0, -1, 0]


def test_recurrence_forgets_at_minus_infinity():
    rng = np.random.default_rng(3)
    q, k, v, dy = (rng.normal(size=(1, 9, 2)) for _ in range(4))
    g = -rng.uniform(0, 1, size=(1, 9, 2))
    g[:, 4] = -np.inf
    y, s, _ = model_ref.glr(q, k, v, g)
    y2, s2, _ = model_ref.glr(q[:, 4:], k[:, 4:], v[:, 4:], g[:, 4:])
    np.testing.assert_array_equal(y[:, 4:], y2)
    grads = model_ref.glr_grads(dy, q, k, v, g)
    assert all(np.isfinite(d).all() for d in grads) and (grads[3][:, 4] == 0).all()


def test_adamw_of_a_constant_gradient_moves_by_the_learning_rate():
    """m / (1 - b1^t) = g and v / (1 - b2^t) = g^2 at every step."""
    p, m, v = np.ones(3), np.zeros(3), np.zeros(3)
    g = np.array([1.0, -2.0, 1e-3])
    for step in range(1, 6):
        p, m, v = model_ref.adamw(p, g, m, v, 0.01, step, eps=0.0)
    np.testing.assert_allclose(p, 1 - 0.05 * np.sign(g), rtol=1e-12)


def test_cross_entropy_gradients_match_differences():
    rng = np.random.default_rng(7)
    x, w = rng.normal(size=(5, 4)), rng.normal(size=(6, 4))
    target, dloss = np.array([0, 5, -100, 2, 6]), rng.normal(size=5)

    def loss():
        return (model_ref.xent(x, w, target)[0] * dloss).sum()

    for got, at in zip(model_ref.xent_grads(dloss, x, w, target), (x, w)):
        np.testing.assert_allclose(got, difference(loss, at), rtol=1e-6, atol=1e-7)
    assert model_ref.xent(x, w, target)[0][2] == 0 == model_ref.xent(x, w, target)[0][4]


def test_cross_entropy_of_equal_logits():
    x, w = np.zeros((2, 3)), np.ones((10, 3))
    loss, lse, _ = model_ref.xent(x, w, np.array([3, 4]))
    np.testing.assert_allclose(loss, np.log(10))
