"""Gradients of a sliding window at scores of millions, where the roundings of a score and of its row's lse are whole powers of e (needs a GPU)."""
import numpy as np
import pytest

from paper_2605_25451_amd import binding as bm
from tests.test_gpu_window import Window, host, pack, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dh,heads,seqs,window,sinks", [
    (128, 4, pack(300, 77), 60, 0), (128, 16, pack(2100), 530, 0), (128, 16, pack(2100), 530, 90), (72, 4, pack(300, 77), 60, 3), (64, 4, pack(300, 77), 60, 3)],
    ids=["pairs", "256 keys", "256 keys, first ones", "72", "64"])
def test_scores_of_millions_have_finite_gradients(dh, heads, seqs, window, sinks):
    """Keys that are the queries themselves: a query's own key has about |q|^2 / sqrt(dh) = 4e7, all others millions less, so the softmax is 1 for it and
    0 for the others; o = v, dP = delta and dS = 0 but for roundings."""
    import torch
    x = Window("bf16", heads, heads, dh, seqs, window, sinks, seed=21)
    rng = np.random.default_rng(22)
    x.q = rounded(2048 * rng.choice([-1.0, 1.0], x.q.shape) * rng.uniform(0.9, 1.1, (x.Tq, heads, 1)), "bf16")
    x.k = x.q.copy()
    x.v, x.d_o = (rng.integers(-4, 5, x.v.shape).astype(np.float64) for _ in range(2))
    o, lse = x.forward()
    assert torch.isfinite(lse[:heads * x.Tq]).all()
    for (a, _) in x.each():
        for h in range(heads):
            s = x.q[a, h] @ x.k[a, h].T * dh ** -0.5
            own = np.diagonal(s).copy()
            s[np.diag_indices_from(s)] = -np.inf
            assert (s.max(1) < own - 1e6).all()
    # o: a weight that bf16 rounds over one that it does not, and the quotient rounded again
    assert (np.abs(host(o)[:x.Tq].reshape(x.v.shape) - x.v) <= 1.01 * 2.0 ** -7 * np.abs(x.v)).all()
    grads = [torch.full((x.Tq, heads * dh), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(3)]
    head, offsets = x.common()
    n = bm.window_attention_backward_scratch_bytes(*x.sizes())
    d_o = x.rows(x.d_o)
    bm.window_attention_backward(*head, o, d_o, lse, *offsets, grads[0], heads * dh, grads[1], grads[2], heads * dh, x.scratch(n), n)
    for g, what in zip(grads, ("dq", "dk", "dv")):
        assert torch.isfinite(g.float()).all(), what
    if dh > 64:
        # a probability of at most 1 times dP - delta, which is what o is off by, and the roundings of both sums of dh products
        ds = (1.01 * 2.0 ** -7 + 2 * dh * 2.0 ** -24) * (np.abs(x.d_o) * np.abs(x.v)).sum(-1, keepdims=True)
        bound = 1.02 * dh ** -0.5 * ds * np.abs(x.k)
        assert (np.abs(host(grads[1]).reshape(x.k.shape)) <= bound).all()
