"""Gradients of a sliding window whose workgroups do not fit a grid are refused before anything is launched (no GPU)."""
import numpy as np
import pytest

from paper_2605_25451_amd import binding as bm

A = [(i + 1) << 40 for i in range(12)]                      # addresses that are never followed, farther apart than any tensor
Q, K, V, O, D_O, LSE, CU, DQ, DK, DV, WORK = A[:11]


@pytest.mark.parametrize("window,sinks", [(65, 0), (300, 4), (1 << 30, 100)])
@pytest.mark.parametrize("own_keys", [False, True])
def test_gradients_of_too_many_tiles_are_refused(window, sinks, own_keys):
    """Within the limits of rows x heads (2^26) and sequences x heads (2^22): 64 heads of 128, all sequences of one token but for one.  Key tiles: 65534
    + 7657 of 128, query tiles: 65534 + 3829 of 256 and as many heads, 1.09 x 2^32 threads in workgroups of 512."""
    S, heads, dh = 65535, 64, 128
    cu = np.arange(S + 1, dtype=np.int32)
    cu[-1] += 980000 - 1
    assert S * heads < 1 << 22 and int(cu[-1]) * heads < 1 << 26
    keys = (K, K, cu[:-1], cu[1:]) if own_keys else (None,) * 4
    ld = heads * dh
    with pytest.raises(bm.BmError) as e:
        bm.window_attention_backward(0, window, sinks, heads, heads, dh, Q, ld, K, V, ld, O, D_O, LSE, CU, cu, *keys, S, DQ, ld, DK, DV, ld, WORK,
                                     1 << 45, stream=0)
    assert e.value.status == bm.BM_ERR_INVALID_ARG and "grid" in bm.last_error()
