"""Pins of the oracle of the embedding and the cross entropy: hand-worked values, identities and central differences."""
import numpy as np
import pytest

from oracle import language_ends as E


def test_worked_values():
    """Two classes with logits 0 and log 3: probabilities 1/4 and 3/4."""
    h, table = np.array([[1.0]]), np.array([[0.0], [np.log(3.0)]])
    r = E.cross_entropy(h, table, [1])
    assert np.isclose(r["lse"][0], np.log(4.0)) and np.isclose(r["loss"][0], np.log(4.0 / 3.0)) and r["best"][0] == 1
    g = E.cross_entropy_backward(h, table, [0], [2.0])
    assert np.allclose(g["dz"], [[2.0 * (0.25 - 1.0), 2.0 * 0.75]])
    assert np.allclose(g["dtable"], [[-1.5], [1.5]]) and np.allclose(g["dh"], [[1.5 * np.log(3.0)]])


def test_cap_limits():
    """A wide cap leaves the logits, a tight one squashes them to +-cap."""
    rng = np.random.default_rng(0)
    h, table = rng.normal(size=(4, 6)), rng.normal(size=(9, 6))
    free, wide = (E.cross_entropy(h, table, [0, 1, 2, 3], c) for c in (0.0, 1e6))
    assert np.allclose(free["loss"], wide["loss"], rtol=1e-9)
    l, z = E.logits(1e6 * h, table, 2.0)
    assert np.allclose(np.abs(l), 2.0) and (np.sign(l) == np.sign(z)).all()


def test_what_does_not_count():
    rng = np.random.default_rng(1)
    h, table = rng.normal(size=(5, 3)), rng.normal(size=(7, 3))
    t = np.array([3, -1, 7, 100, 0])
    assert (E.cross_entropy(h, table, t)["loss"][1:4] == 0).all()
    g = E.cross_entropy_backward(h, table, t, np.ones(5), 4.0)
    assert (g["dh"][1:4] == 0).all() and np.allclose(g["dtable"], E.cross_entropy_backward(h[[0, 4]], table, t[[0, 4]], np.ones(2), 4.0)["dtable"])
    assert (E.embedding(table, t)[1:4] == 0).all() and (E.embedding(table, t, 2.0)[0] == 2 * table[3]).all()


@pytest.mark.parametrize("cap", [0.0, 3.0])
def test_gradients_against_differences(cap):
    rng = np.random.default_rng(2)
    h, table, t, up = rng.normal(size=(4, 5)), rng.normal(size=(6, 5)), np.array([5, 0, -1, 2]), rng.normal(size=4)
    g = E.cross_entropy_backward(h, table, t, up, cap)

    def loss(a, b):
        return float(up @ E.cross_entropy(a, b, t, cap)["loss"])

    for name, x in (("dh", h), ("dtable", table)):
        for i in np.ndindex(*x.shape):
            step = np.zeros_like(x)
            step[i] = 1e-5
            d = (loss(h + step, table) - loss(h - step, table)) if name == "dh" else (loss(h, table + step) - loss(h, table - step))
            assert abs(d / 2e-5 - g[name][i]) < 1e-8, (name, i)


def test_embedding_gradient_is_the_transpose():
    """<dy, embedding(E)> = <embedding_backward(dy), E>, and a base is added to."""
    rng = np.random.default_rng(3)
    table, t, dy = rng.normal(size=(6, 4)), np.array([5, 0, -1, 5, 9, 5]), rng.normal(size=(6, 4))
    grad, size, count = E.embedding_backward(t, dy, 6, 1.5)
    assert np.isclose((dy * E.embedding(table, t, 1.5)).sum(), (grad * table).sum()) and count[5, 0] == 3
    assert np.allclose(E.embedding_backward(t, dy, 6, 1.5, table)[0], grad + table) and (size >= np.abs(grad) - 1e-12).all()
