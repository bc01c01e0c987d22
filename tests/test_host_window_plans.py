"""Which kernels attention with a sliding window takes (host only, no GPU)."""
import numpy as np
import pytest

from paper_2605_25451_amd import binding as bm


def plan(lens, window=100, sinks=0, Hq=32, Hkv=8, dh=128, dtype=0, queries=None):
    """Sequences one behind the other; queries: of each, all tokens unless given."""
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    if queries is None:
        return bm.probe_window_plan(dtype, window, sinks, Hq, Hkv, dh, cu)
    q = np.concatenate([[0], np.cumsum(queries)]).astype(np.int32)
    return bm.probe_window_plan(dtype, window, sinks, Hq, Hkv, dh, q, cu[:-1], cu[1:])


def test_kind_of_the_forward_pass():
    assert plan([500])[0] == (1, 0, 0, 0)
    assert plan([500], dtype=1) == ((0, 0, 0, 0), (0, 0, 0, 0))
    assert plan([500], dh=32)[0][0] == 0
    assert plan([500, 600], queries=[8, 1])[0][0] == plan([500], dtype=1, queries=[8])[0][0] == 2       # 8 rows x 4 heads of a group
    assert plan([500, 600], queries=[9, 1])[0][0] == 1 and plan([500], dtype=1, queries=[9])[0][0] == 0
    assert plan([500], Hq=33, Hkv=1, queries=[1])[0][0] == 1


def test_parts_of_few_queries():
    assert plan([8192], window=1 << 20, queries=[1])[0] == (2, 256, 0, 0)            # 256 tiles of 32 keys, 8 to a part, 8 kv heads
    assert plan([32] * 260, queries=[1] * 260)[0] == (2, 2080, 0, 1)                 # the chip full many times: kv heads on one XCD
    assert plan([500], dh=72, Hq=16, Hkv=16, queries=[1])[0][3] == 1                 # rows of a head that are no whole cache lines
    assert plan([4096] * 8, window=1 << 20, queries=[1] * 8)[0][2] == 1              # 134 MB of keys and values
    assert plan([4096] * 3, window=1 << 20, queries=[1] * 3)[0][2] == 0              # 50
    assert plan([4096] * 8, window=512, queries=[1] * 8)[0][2] == 0                  # 17 that are visible
    assert plan([4096] * 8, window=1 << 20, dtype=1, dh=64, queries=[1] * 8)[0][2] == 1
    assert plan([4096] * 8, window=1 << 20, dtype=1, dh=64, queries=[2] * 8)[0][2] == 0      # 8 rows: read by two workgroups


def streamed(spans, **kw):
    """Single queries behind keys begin .. end; none where there are no keys."""
    args = dict(dtype=0, window=1 << 20, sinks=0, Hq=32, Hkv=8, dh=128, **kw)
    begin, end = np.array(spans, np.int32).T
    return bm.probe_window_plan(*args.values(), np.concatenate([[0], np.cumsum(end > begin)]), begin, end)[0][2]


def test_keys_of_several_sequences_stay_in_the_caches():
    slots = [(i * 5000, i * 5000 + 4096) for i in range(64)]
    rng = np.random.default_rng(1)
    assert streamed(slots) == streamed(slots[::-1]) == streamed([slots[i] for i in rng.permutation(64)]) == 1
    assert streamed([(7, 7)] + slots + [(0, 0)]) == 1                                # sequences of no keys own nothing
    assert streamed([(0, 4096)] * 64) == 0
    answers = [slots[i // 4] for i in range(64)]                                     # four answers to a question each
    assert streamed(answers) == streamed([answers[i] for i in rng.permutation(64)]) == 0
    assert streamed(slots[:-1] + [(10 * 5000 + 100, 10 * 5000 + 4000)]) == streamed(slots[1:] + [(0, 5001)]) == 0
    many = [(i * 300, i * 300 + 256) for i in range(4000)]
    many = [many[i] for i in rng.permutation(4000)]
    assert streamed(many) == 1 and streamed(many[:-1] + many[:1]) == 0
    assert streamed(many[:-1] + [(many[0][0] + 255, many[0][0] + 300)]) == 0


@pytest.mark.parametrize("args,want", [
    (dict(lens=[8192], window=2048, sinks=64), (256, 256, 1, 8 * 4)),                # first keys in parts of 2048 rows
    (dict(lens=[8192], window=64), (128, 128, 2, 0)), (dict(lens=[8192], window=65), (128, 256, 1, 0)),
    (dict(lens=[8192], window=255), (128, 256, 1, 0)), (dict(lens=[8192], window=256), (256, 256, 1, 0)),
    (dict(lens=[1000], window=64, Hq=16, Hkv=16), (128, 256, 1, 0)),                 # 128 tiles of queries: dQ stays beside dK/dV
    (dict(lens=[777], window=300, Hq=16, Hkv=16), (128, 256, 1, 0)),                 # 64 workgroups of 256 keys
    (dict(lens=[300], window=20, sinks=3, Hq=4, Hkv=4, dh=64), (128, 128, 1, 2 * 4)),
    (dict(lens=[300], window=20, sinks=3, Hq=4, Hkv=4, dh=72), (128, 128, 1, 2 * 4))])
def test_tiles_of_the_gradients(args, want):
    assert plan(**args)[1] == want


def test_plan_refusals():
    for bad in (dict(window=0), dict(Hq=3), dict(sinks=129), dict(lens=[5], queries=[6])):
        with pytest.raises(bm.BmError):
            plan(**{"lens": [500], **bad})
    with pytest.raises(bm.BmError):
        bm._check(bm.lib().bm_probe_window_plan(0, 5, 0, 1, 1, 64, None, None, None, 1, None, None))
