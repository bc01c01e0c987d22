"""The loss over the whole range of finite logits (needs a GPU)."""
import numpy as np
import pytest

from tests.test_gpu_train import NAMES, TYPES, check_loss, cross_entropy, device, ints

pytestmark = pytest.mark.gpu


def sizes(rng, V, dtype):
    """Rows of every kind around magnitudes from where the products with log2 e are whole numbers to where fp32 ends."""
    rows = []
    for size in (3e6, 1.1e7, 1.3e7, 1e8, 2e9, 1e10, 1e20, 1e30, 9e37):
        for sign in (1, -1):
            m = sign * size
            rows.append(np.full(V, m))                                # one value throughout: a uniform distribution
            rows.append(m * rng.uniform(0.5, 1.0, V))                 # words far apart
            near = np.full(V, m)                                      # words a few steps of the type apart
            near += np.abs(m) * rng.integers(-2, 3, V) * 2.0 ** (-7 if dtype == 0 else -23)
            rows.append(near)
            some = rng.standard_normal(V)                             # one word in ten of that size, a mask for instance
            some[rng.random(V) < 0.1] = m
            rows.append(some)
    return np.stack(rows)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("V", [1, 5, 300, 8000, 16000, 33000, 66003])
def test_finite_logits_of_any_size(V, dtype):
    """In every kernel of whole rows (by V and by T) and in parts of rows (few of them)."""
    import torch
    rng = np.random.default_rng(V)
    logits, z64 = device(sizes(rng, V, dtype), dtype)
    T = len(z64)
    labels = rng.integers(0, V, T)
    first = np.arange(T) % 3 == 0
    labels[first] = z64[first].argmax(axis=1)
    runs = [(0, T), (0, 20), (20, 52)]
    for a, b in runs:
        z, lab = logits[a:b].clone(), ints(labels[a:b])
        grad = torch.full_like(z, 9.0)
        loss = cross_entropy(dtype, b - a, V, z, V, lab, None, grad, V).double().cpu().numpy()
        check_loss(loss, grad.double().cpu().numpy(), z64[a:b], labels[a:b], None, dtype)
        again = cross_entropy(dtype, b - a, V, z, V, lab, None, z, V).double().cpu().numpy()       # in place
        assert np.array_equal(again, loss) and torch.equal(z, grad)
    if V == 16000:                                                    # more rows than there are CUs twice over
        z = logits.repeat(10, 1)
        grad = torch.empty_like(z)
        loss = cross_entropy(dtype, 10 * T, V, z, V, ints(np.tile(labels, 10)), None, grad, V).view(10, T)
        assert torch.equal(loss, loss[:1].expand(10, T)) and torch.equal(grad.view(10, T, V), grad.view(10, T, V)[:1].expand(10, T, V))
        check_loss(loss[0].double().cpu().numpy(), grad[:T].double().cpu().numpy(), z64, labels, None, dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("mask", [-1e9, -1e10, -1e30, -3.3e38, -np.inf])
@pytest.mark.parametrize("V", [300, 5000, 16000, 33000, 66003])
def test_words_of_a_row_masked_in_a_run(V, mask, dtype):
    """A thread then holds masked words alone, or holds them before any other."""
    import torch
    rng = np.random.default_rng(V)
    z = rng.standard_normal((40, V))
    runs = [(0, V // 2), (V // 2, V), (0, V - 1), (1, V), (V // 3, 2 * V // 3), (0, 64), (V - 64, V), (8, 264)]
    for t in range(40):
        a, b = runs[t % len(runs)]
        z[t, a:b] = mask
    labels = np.array([rng.choice(np.nonzero(row != mask)[0]) for row in z])
    logits, z64 = device(z, dtype)
    grad = torch.full_like(logits, 9.0)
    loss = cross_entropy(dtype, 40, V, logits, V, ints(labels), None, grad, V).double().cpu().numpy()
    check_loss(loss, grad.double().cpu().numpy(), z64, labels, None, dtype)
