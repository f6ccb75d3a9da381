"""The oracle of a model's ends and of Newton-Schulz updates, against definitions of another kind: hand-worked
numbers, central differences, singular values."""
import numpy as np

import oracle.model_oracle as M


def test_embed_by_hand():
    table = np.array([[1.0, 2.0], [3.0, -4.0], [0.5, 0.0]])
    ids = np.array([1, -1, 2, 1, 3])
    assert np.array_equal(M.embed(table, ids, 2.0), [[6, -8], [0, 0], [1, 0], [6, -8], [0, 0]])
    grad, size, n = M.embed_backward(ids, np.array([[1.0, 1], [9, 9], [2, -2], [3, -5], [9, 9]]), 3, 0.5)
    assert np.array_equal(grad, [[0, 0], [2, -2], [1, -1]])
    assert np.array_equal(size, [[0, 0], [2, 3], [1, 1]]) and np.array_equal(n, [0, 2, 1])


def test_loss_by_hand():
    x, w = np.array([[1.0, 0.0], [0.0, 2.0]]), np.array([[np.log(2.0), 0.0], [0.0, np.log(3.0) / 2], [0.0, 0.0]])
    loss, lse = M.head_loss(x, w, [0, 3], 1.0)          # exp of the logits: (2, 1, 1) and (1, 3, 1)
    assert np.allclose(lse, [np.log(4.0), np.log(5.0)]) and np.allclose(loss, [np.log(2.0), 0.0])
    r = M.head_slope(x, w, [0, 3], [1.0, 1.0], 1.0)
    assert np.allclose(r, [[-0.5, 0.25, 0.25], [0, 0, 0]])


def test_head_gradients_against_differences():
    rng = np.random.default_rng(0)
    x, w = rng.normal(size=(5, 4)), rng.normal(size=(7, 4))
    targets, dloss = np.array([6, 0, -1, 3, 7]), rng.normal(size=5)
    dx, dw = M.head_backward(x, w, targets, dloss, 0.7)
    f = lambda x, w: (M.head_loss(x, w, targets, 0.7)[0] * dloss).sum()   # noqa: E731
    for _ in range(5):
        a, b = rng.normal(size=x.shape), rng.normal(size=w.shape)
        h = 1e-5
        assert abs((f(x + h * a, w) - f(x - h * a, w)) / (2 * h) - (dx * a).sum()) < 1e-8
        assert abs((f(x, w + h * b) - f(x, w - h * b)) / (2 * h) - (dw * b).sum()) < 1e-8


def test_newton_schulz_acts_on_singular_values():
    rng = np.random.default_rng(1)
    coef = (3.4445, -4.7750, 2.0315)
    for shape in ((6, 9), (9, 6), (5, 5), (1, 7)):
        g = rng.normal(size=shape)
        u, s, v = np.linalg.svd(g, full_matrices=False)
        s = s / np.sqrt((s * s).sum())
        for _ in range(5):
            s = coef[0] * s + coef[1] * s ** 3 + coef[2] * s ** 5
        x, norms = M.newton_schulz(g, 5, *coef, 0.0)
        assert np.allclose(x, (u * s) @ v, atol=1e-12) and len(norms) == 6
        assert np.isclose(norms[0], 1.0) and np.isclose(norms[-1], np.sqrt((s * s).sum()))
