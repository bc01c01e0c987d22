"""The oracle of the training-step operators against what defines them: differences of the functions
whose gradients they are, and closed forms."""
import numpy as np

from oracle import train_oracle as to


def test_embedding_gradient_is_that_of_the_lookup():
    rng = np.random.default_rng(0)
    table, ids = rng.standard_normal((5, 3)), np.array([2, -1, 4, 2, 0, 2])
    dy, y0 = rng.standard_normal((6, 3)), np.zeros((6, 3))
    got = to.embedding_backward(dy, ids, 1.7, np.zeros((5, 3)))
    f = lambda t: (to.embedding_forward(t, ids, 1.7, y0) * dy).sum()
    for v in range(5):
        for c in range(3):
            up = table.copy()
            up[v, c] += 1.0                                  # linear: a difference of any size is exact
            assert abs(f(up) - f(table) - got[v, c]) < 1e-12


def test_embedding_leaves_other_rows_alone():
    y = to.embedding_forward(np.ones((2, 2)), [-1, 1, 2], 3.0, np.full((3, 2), 9.0))
    assert (y[0] == 9).all() and (y[1] == 3).all() and np.isnan(y[2]).all()
    g = to.embedding_backward(np.ones((3, 2)), [-1, 1, 2], 3.0, np.full((2, 2), 5.0))
    assert (g == [[5, 5], [8, 8]]).all()


def test_cross_entropy_against_differences():
    rng = np.random.default_rng(1)
    z, labels, w = 3 * rng.standard_normal((4, 7)), np.array([3, -1, 0, 6]), np.array([0.5, 9.0, 1.0, 2.0])
    loss, grad = to.cross_entropy(z, labels, w)
    assert loss[1] == 0 and (grad[1] == 0).all()
    h = 1e-6
    for t in range(4):
        for v in range(7):
            up, dn = z.copy(), z.copy()
            up[t, v] += h
            dn[t, v] -= h
            d = (to.cross_entropy(up, labels, w)[0].sum() - to.cross_entropy(dn, labels, w)[0].sum()) / (2 * h)
            assert abs(d - grad[t, v]) < 1e-8


def test_cross_entropy_closed_forms():
    loss, grad = to.cross_entropy(np.zeros((1, 8)), [5])
    assert abs(loss[0] - np.log(8)) < 1e-15 and abs(grad[0, 5] + 7 / 8) < 1e-15
    z = np.array([[-np.inf, 1.0, 1.0]])
    loss, grad = to.cross_entropy(z, [1])
    assert abs(loss[0] - np.log(2)) < 1e-15 and grad[0, 0] == 0
    assert np.isnan(to.cross_entropy(z, [3])[0][0])


def test_orthogonalize_moves_singular_values_by_the_polynomial():
    rng = np.random.default_rng(2)
    for shape in ((5, 9), (9, 5), (1, 4), (6, 6)):
        G = rng.standard_normal(shape)
        u, s, v = np.linalg.svd(G, full_matrices=False)
        s = s / (np.sqrt((s * s).sum()) + np.float32(1e-7))
        a, b, c = (float(np.float32(x)) for x in (3.4445, -4.775, 2.0315))
        for _ in range(4):
            s = a * s + b * s ** 3 + c * s ** 5
        X = to.orthogonalize(G, (3.4445, -4.775, 2.0315), 4, 1e-7)[-1]
        want = (u * s) @ v
        assert np.abs((X.T if shape[0] > shape[1] else X) - want).max() < 1e-12


def test_orthogonalize_converges_to_an_orthogonal_matrix():
    G = np.random.default_rng(3).standard_normal((6, 11))
    X = to.orthogonalize(G, (1.875, -1.25, 0.375), 30, 0.0)[-1]
    assert np.abs(X @ X.T - np.eye(6)).max() < 1e-12
