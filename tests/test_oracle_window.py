"""The oracle of rotations over several axes and of sliding windows against what defines them: differences of the functions
whose gradients they are, and closed forms."""
import numpy as np
import pytest

from oracle import block_oracle as bo
from oracle import window_oracle as wo


def difference(f, x, h=1e-6):
    g = np.zeros(x.shape)
    for i in np.ndindex(x.shape):
        up, dn = x.copy(), x.copy()
        up[i] += h
        dn[i] -= h
        g[i] = (f(up) - f(dn)) / (2 * h)
    return g


def test_angles_by_axis():
    pos = np.array([[3, 0], [5, 7], [0, 2]])
    a = wo.angles(pos, [1, 0, 3], 100.0)
    assert a.shape == (2, 4)
    np.testing.assert_allclose(a[0], [3.0, 0.0, 0.0, 0.0])
    np.testing.assert_allclose(a[1], [0.0] + [2 * 100.0 ** -(i / 4) for i in (1, 2, 3)])
    own = wo.angles(pos, [2, 2], 100.0, own_frequencies=True)
    np.testing.assert_allclose(own, [[3, 0.3, 5, 0.5], [0, 0, 7, 0.7]])


def test_turn_is_a_rotation_and_depends_on_the_distance_of_positions():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 8))
    at = lambda p: wo.angles(np.array(p)[:, None], [1, 1, 2], 50.0)
    z = wo.turn(q, at([4, 9, 2]))
    assert abs((z * z).sum() - (q * q).sum()) < 1e-12
    np.testing.assert_allclose(wo.turn(z, at([4, 9, 2]), -1.0), q, atol=1e-14)
    dot = lambda p, r: (wo.turn(q, at(p)) * wo.turn(k, at(r))).sum()
    assert abs(dot([4, 9, 2], [1, 3, 2]) - dot([14, 29, 102], [11, 23, 102])) < 1e-12


def test_one_axis_is_the_rotation_of_a_block():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 2, 16))
    got = wo.turn(x, wo.angles(np.arange(5)[None], [8], 10000.0))
    np.testing.assert_allclose(got, bo.rope_apply(x, bo.rope_angles(np.arange(5), 16, 10000.0)), atol=1e-12)


@pytest.mark.parametrize("norm", [False, True])
def test_rotary_gradient_against_differences(norm):
    rng = np.random.default_rng(2)
    x, dz = rng.standard_normal((2, 3, 2, 8))
    a = wo.angles(rng.integers(-9, 9, (2, 3)), [3, 1], 30.0)
    gain = rng.standard_normal(8) if norm else None
    dx, dg = wo.rotary_backward(x, a, dz, gain, 1e-3)
    f = lambda x_, g_: (wo.rotary_forward(x_, a, g_, 1e-3) * dz).sum()
    np.testing.assert_allclose(dx, difference(lambda t: f(t, gain), x), atol=1e-8)
    if norm:
        np.testing.assert_allclose(dg, difference(lambda t: f(x, t), gain), atol=1e-8)


def test_visible_by_hand():
    assert (wo.visible(4, 4, 2, 1) == [[1, 0, 0, 0], [1, 1, 0, 0], [1, 1, 1, 0], [1, 0, 1, 1]]).all()
    assert (wo.visible(1, 5, 2, 0) == [[0, 0, 0, 1, 1]]).all()
    assert (wo.visible(3, 3, 100, 0) == np.tri(3)).all() and (wo.visible(3, 3, 1, 100) == np.tri(3)).all()
    assert (wo.visible(3, 3, 1, 0) == np.eye(3)).all()


def test_attention_closed_forms():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((6, 4, 8)), rng.standard_normal((6, 2, 8)), rng.standard_normal((6, 2, 8))
    o, lse = wo.attention(q, k, v, 1, 0)                     # each query sees its own key
    np.testing.assert_allclose(o, np.repeat(v, 2, axis=1))
    o, lse = wo.attention(np.zeros((6, 4, 8)), k, v, 2, 1)   # equal weights
    np.testing.assert_allclose(o[5, 3], (v[0, 1] + v[4, 1] + v[5, 1]) / 3)
    np.testing.assert_allclose(lse[:, 5], np.log(3))
    # the last queries alone are the last rows of all of them
    all_o, all_lse = wo.attention(q, k, v, 3, 1)
    o, lse = wo.attention(q[4:], k, v, 3, 1)
    np.testing.assert_allclose(o, all_o[4:])
    np.testing.assert_allclose(lse, all_lse[:, 4:])


@pytest.mark.parametrize("Lq,window,sinks", [(7, 3, 0), (7, 2, 2), (3, 2, 1), (7, 50, 0)])
def test_attention_gradient_against_differences(Lq, window, sinks):
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((Lq, 2, 4)), rng.standard_normal((7, 1, 4)), rng.standard_normal((7, 1, 4))
    d_o = rng.standard_normal(q.shape)
    dq, dk, dv = wo.attention_backward(q, k, v, d_o, window, sinks)
    f = lambda a, b, c: (wo.attention(a, b, c, window, sinks)[0] * d_o).sum()
    np.testing.assert_allclose(dq, difference(lambda t: f(t, k, v), q), atol=1e-8)
    np.testing.assert_allclose(dk, difference(lambda t: f(q, t, v), k), atol=1e-8)
    np.testing.assert_allclose(dv, difference(lambda t: f(q, k, t), v), atol=1e-8)
