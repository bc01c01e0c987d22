"""The loss over the whole range of finite logits, and of rows that a model is sure of (needs a GPU)."""
import numpy as np
import pytest

from tests.test_gpu_train import F, NAMES, TYPES, check_loss, cross_entropy, device, ints

pytestmark = pytest.mark.gpu


def check_by_difference(loss, z64, labels):
    """loss = (max - z[label]) + log s with s = sum of exp(z - max): a bound that does not know how large the logits are.

    A term of s is off by its share of what its difference, the factor log2 e and the function round (3 |z - max| + 6), the sum by a
    thread's additions and the joins (3 V/256 + 64).  max - z[label] is rounded once, log s by its own function, the factor log 2, the
    difference to the rounding of max * log2 e (at most a half) and their sum: 8 of each are more than all of these."""
    top = z64.max(axis=1)
    with np.errstate(over="ignore"):
        away = top[:, None] - z64
    p = np.exp(-away)
    S = p.sum(axis=1)
    share = (p / S[:, None] * (3 * np.minimum(away, 110.0) + 6)).sum(axis=1)
    ahead = top - z64[np.arange(len(z64)), labels]
    want = ahead + np.log(S)
    bound = (share + 3 * -(-z64.shape[1] // 256) + 64 + 8 * (ahead + np.log(S) + 1)) * F
    off = np.abs(loss - want)
    assert (off <= bound).all(), (np.argmax(off - bound), np.max(off / bound))


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
        check_by_difference(loss, z64[a:b], labels[a:b])
        again = cross_entropy(dtype, b - a, V, z, V, lab, None, z, V).double().cpu().numpy()       # in place
        assert np.array_equal(again, loss) and torch.equal(z, grad)
    if V == 16000:                                                    # more rows than there are CUs twice over
        z = logits.repeat(10, 1)
        grad = torch.empty_like(z)
        loss = cross_entropy(dtype, 10 * T, V, z, V, ints(np.tile(labels, 10)), None, grad, V).view(10, T)
        assert torch.equal(loss, loss[:1].expand(10, T)) and torch.equal(grad.view(10, T, V), grad.view(10, T, V)[:1].expand(10, T, V))
        check_loss(loss[0].double().cpu().numpy(), grad[:T].double().cpu().numpy(), z64, labels, None, dtype)
        check_by_difference(loss[0].double().cpu().numpy(), z64, labels)


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("V", [1, 7, 300, 5000, 33000, 66003])
def test_loss_of_rows_a_model_is_sure_of(V, dtype):
    """The label 12 to 20 ahead of the other words, wherever the logits lie."""
    import torch
    rng = np.random.default_rng(V)
    T = 160
    labels = rng.integers(0, V, T)
    z = 0.5 * rng.standard_normal((T, V))
    z[np.arange(T), labels] = rng.uniform(12, 20, T)
    z += np.repeat([0.0, 100.0, -100.0, 1000.0, -1000.0], T // 5)[:, None]
    order = rng.permutation(T)
    logits, z64 = device(z[order], dtype)
    labels = labels[order]
    runs = [(0, T), (0, 30)]
    for a, b in runs:
        grad = torch.empty_like(logits[a:b])
        loss = cross_entropy(dtype, b - a, V, logits[a:b].contiguous(), V, ints(labels[a:b]), None, grad, V).double().cpu().numpy()
        check_loss(loss, grad.double().cpu().numpy(), z64[a:b], labels[a:b], None, dtype)
        check_by_difference(loss, z64[a:b], labels[a:b])


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
    check_by_difference(loss, z64, labels)
