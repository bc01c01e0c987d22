"""Kernels of the windowed attention and of the rotation that only certain sizes take, each case with a look at the plan that it is meant to reach (needs a
GPU).  Classes and tolerances of test_gpu_window.py."""
import numpy as np
import pytest

from paper_2605_25451_amd import binding as bm
from tests.test_gpu_window import Rotary, Window, dev, pack

pytestmark = pytest.mark.gpu


def plan(x):
    Hq, Hkv, dh = x.heads
    own = (x.begin, x.end) if x.own else ()
    return bm.probe_window_plan(x.code, x.window, x.sinks, Hq, Hkv, dh, x.cu, *own)


def both(x):
    x.check_forward(*x.forward())
    x.check_backward(*x.backward())


@pytest.mark.parametrize("window,sinks", [(1, 0), (17, 90), (64, 5)])
@pytest.mark.parametrize("heads,seqs", [((16, 4), [(1 + i * 53 % 260,) * 2 for i in range(40)]), ((16, 8), [(1 + i * 53 % 260, 7 + i * 97 % 700 + 260) for i in range(40)]),
                                        ((8, 2), [(1 + i * 53 % 260,) * 2 for i in range(80)]), ((8, 8), [(i * 53 % 260, 3 + i * 97 % 700 + 260) for i in range(80)])],
                         ids=["40", "40 behind others", "80", "80 behind others"])
def test_queries_gradients_in_a_launch_of_their_own(heads, seqs, window, sinks):
    """Narrow windows at head size 128 with two tiles of 128 queries and more for every CU; packs with and without a table of their tiles."""
    x = Window("bf16", *heads, 128, seqs, window, sinks, seed=31, gap=2 if seqs[0][0] != seqs[0][1] else None)
    assert plan(x)[1][:3] == (128, 128, 2)
    both(x)


@pytest.mark.parametrize("window,sinks", [(60, 5), (64, 0)])
def test_queries_gradients_of_a_long_sequence_in_a_launch_of_their_own(window, sinks):
    """First keys in parts next to it."""
    x = Window("bf16", 32, 8, 128, pack(2100), window, sinks, seed=32)
    assert plan(x)[1] == (128, 128, 2, 5 * 32 if sinks else 0)       # q heads of a group one by one
    both(x)


@pytest.mark.parametrize("sinks", [0, 5, 90])
@pytest.mark.parametrize("behind", [0, 140])
def test_wide_key_tiles_of_many_sequences(sinks, behind):
    """256 keys to a workgroup and more sequences than a table holds, a long one among them."""
    lens = [200 + i * 31 % 57 for i in range(80)]
    lens[40] = 1300
    x = Window("bf16", 8, 4, 128, [(n - behind, n) for n in lens], 256, sinks, seed=33, gap=1 if behind else None)
    assert plan(x)[1][:3] == (256, 256, 1) and (plan(x)[1][3] > 0) == (sinks > 0)
    both(x)


STREAMED = [("bf16", 64, 16, 8, 20, 3000), ("bf16", 72, 16, 8, 14, 3500), ("bf16", 128, 8, 4, 16, 2000), ("bf16", 64, 8, 8, 100, 500), ("fp32", 64, 4, 4, 20, 2000),
            ("fp32", 8, 8, 4, 100, 3200)]


@pytest.mark.parametrize("dtype,dh,Hq,Hkv,S,keys", STREAMED)
@pytest.mark.parametrize("window,sinks", [(1 << 20, 0), (2900, 40)])
def test_few_queries_past_the_caches(dtype, dh, Hq, Hkv, S, keys, window, sinks):
    x = Window(dtype, Hq, Hkv, dh, [(1, keys - 3 * (i % 7)) for i in range(S)], window, sinks, seed=34, gap=1)
    assert plan(x)[0][0] == 2 and plan(x)[0][2] == 1
    x.check_forward(*x.forward())


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("fp32", 32)])
def test_few_queries_of_more_workgroups_than_the_chip_holds(dtype, dh):
    """The kv heads of a part on one XCD."""
    x = Window(dtype, 16, 8, dh, [(i * 3 % 4, 3 + i * 37 % 300) for i in range(400)], 200, 6, seed=35, gap=1)
    assert plan(x)[0][0] == 2 and plan(x)[0][1] >= 2048 and plan(x)[0][3] == 1
    x.check_forward(*x.forward())


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("fp32", 32), ("bf16", 32), ("bf16", 16)])
@pytest.mark.parametrize("norm", [False, True])
def test_rotary_of_many_small_heads(dtype, dh, norm):
    """More than 32 MB of heads of 128 bytes, which go past the caches, and of less, which do not."""
    T = 10500 * 64 // dh // (1 if dtype == "bf16" else 2)
    r = Rotary(dtype, norm, T, 12, 12, dh, [dh // 8, dh // 2 - dh // 8], False, seed=36)
    assert T * 24 * dh * (2 if dtype == "bf16" else 4) > 32e6
    r.check_forward(r.forward())
    r.check_backward(*r.backward())


@pytest.mark.parametrize("dh,Hq,Hkv,lens", [(64, 4, 2, (257, 90)), (72, 4, 2, (257, 90)), (128, 4, 2, (257, 90)), (64, 8, 8, (700, 3, 129))])
def test_a_wide_window_has_the_bits_of_causal_attention(dh, Hq, Hkv, lens):
    """Where the causal pass takes tiles of 128 rows as well: the same products in the same order, the same running maxima but for the one before the first
    key, which is forgotten with it."""
    import torch
    x = Window("bf16", Hq, Hkv, dh, pack(*lens), sum(lens), 0, seed=37, scale=3.0)
    assert bm.probe_attention_plan(1, Hq, Hkv, dh, x.cu)[0] == 128
    o, lse = x.forward()
    rows = torch.cat([x.rows(x.q), x.rows(x.k), x.rows(x.v)], 1)
    o2, lse2 = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
    bm.attention_forward(x.code, 1, Hq, Hkv, dh, rows, rows[:, Hq * dh:], rows[:, (Hq + Hkv) * dh:], (Hq + 2 * Hkv) * dh, dev(x.cu), x.cu, len(lens), x.Tq,
                         max(lens), o2, lse2)
    assert torch.equal(o[:x.Tq], o2[:x.Tq]) and torch.equal(lse[:Hq * x.Tq], lse2[:Hq * x.Tq])
