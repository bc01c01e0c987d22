"""What the rotation of queries and keys and the attention of a sliding window refuse, before anything is launched (no GPU)."""
import numpy as np
import pytest

from paper_2605_25451_amd import binding as bm

A = [(i + 1) << 20 for i in range(16)]                      # addresses that are never followed
DESC = dict(dtype=0, n_q_heads=4, n_kv_heads=2, head_dim=16, pairs=[2, 3, 3], base=10000.0, own_frequencies=False, norm=True, eps=1e-6)


def refused(status, fn, *args):
    with pytest.raises(bm.BmError) as e:
        fn(*args, stream=0)
    assert e.value.status == status and bm.last_error()


FORWARD = dict(T=5, q=A[0], k=A[1], ld=64, positions=A[2], q_gain=A[3], k_gain=A[4], q_out=A[5], k_out=A[6], ld_out=64)
BACKWARD = dict(T=5, q=A[0], k=A[1], ld=64, positions=A[2], q_gain=A[3], k_gain=A[4], dq_out=A[5], dk_out=A[6], ld_dout=64, dq=A[7],
                dk=A[8], ld_dqk=64, dq_gain=A[9], dk_gain=A[10], scratch=A[11], scratch_bytes=1 << 30)


def rotary(fn, call, **bad):
    desc = bm.make_qk_rotary_desc(**{**DESC, **{n: v for n, v in bad.items() if n in DESC}})
    return (fn, desc) + tuple({**call, **{n: v for n, v in bad.items() if n in call}}.values())


BAD_DESC = [dict(dtype=2), dict(n_q_heads=-1), dict(n_q_heads=0, n_kv_heads=0), dict(pairs=[2, 3, 2]), dict(pairs=[]),
            dict(pairs=[2, 2, 2, 1, 1]), dict(pairs=[9, -1]), dict(base=0.0), dict(base=-1.0), dict(base=float("nan")),
            dict(base=float("inf")), dict(eps=-1.0), dict(eps=float("nan")), dict(norm=2), dict(own_frequencies=2)]


@pytest.mark.parametrize("bad", BAD_DESC + [
    dict(T=-1), dict(T=(1 << 26) + 1), dict(q=None), dict(k=None), dict(q=A[0] + 2), dict(ld=60), dict(ld=56), dict(positions=None),
    dict(positions=A[2] + 4), dict(q_gain=None), dict(k_gain=A[4] + 8), dict(norm=False), dict(q_out=None), dict(k_out=A[6] + 8),
    dict(ld_out=63), dict(ld_out=48), dict(q_out=A[0], ld_out=72)])
def test_rotary_forward_refusals(bad):
    refused(bm.BM_ERR_INVALID_ARG, *rotary(bm.qk_rotary_forward, FORWARD, **bad))


@pytest.mark.parametrize("bad", BAD_DESC + [
    dict(T=-1), dict(q=None), dict(k=None), dict(ld=60), dict(positions=None), dict(q_gain=None), dict(dk_gain=None), dict(norm=False),
    dict(dq_out=None), dict(dk_out=A[6] + 2), dict(ld_dout=32), dict(dq=None), dict(dk=A[8] + 8), dict(ld_dqk=60), dict(dq=A[5], ld_dqk=72),
    dict(dq=A[0], ld_dqk=72), dict(scratch=A[11] + 8), dict(dq_gain=A[9] + 4)])
def test_rotary_backward_refusals(bad):
    refused(bm.BM_ERR_INVALID_ARG, *rotary(bm.qk_rotary_backward, BACKWARD, **bad))


@pytest.mark.parametrize("head_dim", [0, 4, 12, 20, 264])
def test_rotary_head_sizes(head_dim):
    refused(bm.BM_ERR_UNSUPPORTED, *rotary(bm.qk_rotary_forward, FORWARD, head_dim=head_dim, pairs=[head_dim // 2]))


def test_rotary_workspace():
    desc = bm.make_qk_rotary_desc(**DESC)
    need = bm.qk_rotary_backward_scratch_bytes(desc, 5)
    assert need > 0
    for bad in (dict(scratch_bytes=need - 1), dict(scratch=None), dict(scratch_bytes=0)):
        refused(bm.BM_ERR_WORKSPACE_TOO_SMALL, *rotary(bm.qk_rotary_backward, BACKWARD, **bad))
    assert bm.qk_rotary_backward_scratch_bytes(bm.make_qk_rotary_desc(**{**DESC, "norm": False}), 5) == 0
    assert bm.qk_rotary_backward_scratch_bytes(desc, 0) == bm.qk_rotary_backward_scratch_bytes(desc, -1) == 0
    assert bm.qk_rotary_backward_scratch_bytes(bm.make_qk_rotary_desc(**{**DESC, "pairs": [1]}), 5) == 0


def test_rotary_workspace_is_enough_for_any_tokens():
    for heads in ((32, 8), (4, 0), (1 << 16, 1 << 16)):
        desc = bm.make_qk_rotary_desc(**{**DESC, "n_q_heads": heads[0], "n_kv_heads": heads[1]})
        assert len({bm.qk_rotary_backward_scratch_bytes(desc, T) for T in (1, 7, 100, 2000, 8192, 1 << 26)}) == 1


def test_rotary_of_no_tokens():
    desc = bm.make_qk_rotary_desc(**DESC)
    bm.qk_rotary_forward(desc, 0, None, None, 0, None, None, None, None, None, 0, stream=0)
    bm.qk_rotary_backward(desc, 0, None, None, 0, None, None, None, None, None, 0, None, None, 0, None, None, stream=0)


SIZES = dict(dtype=0, window=8, sinks=2, Hq=4, Hkv=2, dh=64)
CALL = dict(q=A[0], ld_q=256, k=A[1], v=A[2], ld_kv=128, cu_q_dev=A[3], cu_q_host=[0, 3, 5], k_begin_dev=A[4], k_end_dev=A[5],
            k_begin_host=[0, 10], k_end_host=[3, 16], S=2, o=A[6], lse=A[7], scratch=A[8], scratch_bytes=1 << 40)
GRAD = dict(q=A[0], ld_q=256, k=A[1], v=A[2], ld_kv=128, o=A[6], d_o=A[9], lse=A[7], cu_q_dev=A[3], cu_q_host=[0, 3, 5], k_begin_dev=A[4],
            k_end_dev=A[5], k_begin_host=[0, 10], k_end_host=[3, 16], S=2, dq=A[10], ld_dq=256, dk=A[11], dv=A[12], ld_dkv=128,
            scratch=A[8], scratch_bytes=1 << 40)
BAD_WINDOW = [dict(dtype=2), dict(window=0), dict(window=-5), dict(sinks=-1), dict(sinks=129), dict(Hq=3), dict(Hq=0), dict(Hkv=0),
              dict(S=0), dict(ld_q=255), dict(ld_q=252), dict(ld_kv=120), dict(cu_q_dev=None), dict(cu_q_host=None),
              dict(k_begin_dev=None), dict(k_end_host=None), dict(cu_q_host=[1, 3, 5]), dict(cu_q_host=[0, 3, 2]),
              dict(k_end_host=[3, 9]), dict(k_begin_host=[-1, 10]), dict(k_end_host=[2, 16]), dict(k_end_host=[3, 11]),
              dict(cu_q_host=[0, 3, (1 << 28) + 1], k_end_host=[3, 1 << 30]), dict(k=None), dict(v=A[2] + 8), dict(scratch=A[8] + 8),
              dict(Hq=1 << 20, Hkv=1 << 20, ld_q=1 << 26, ld_kv=1 << 26),
              dict(Hq=4096, Hkv=4096, ld_q=1 << 18, ld_kv=1 << 18, cu_q_host=[0, 3, 1 << 24], k_end_host=[3, 1 << 25])]


@pytest.mark.parametrize("bad", BAD_WINDOW + [dict(q=None), dict(o=None), dict(lse=None), dict(o=A[6] + 4)])
def test_window_forward_refusals(bad):
    refused(bm.BM_ERR_INVALID_ARG, bm.window_attention_forward, *{**SIZES, **CALL, **bad}.values())


@pytest.mark.parametrize("bad", BAD_WINDOW + [dict(q=None), dict(o=None), dict(lse=None), dict(d_o=None), dict(dq=None), dict(dk=None),
                                              dict(dv=A[12] + 2), dict(ld_dq=254), dict(ld_dkv=64), dict(ld_dkv=132)])
def test_window_backward_refusals(bad):
    refused(bm.BM_ERR_INVALID_ARG, bm.window_attention_backward, *{**SIZES, **GRAD, **bad}.values())


@pytest.mark.parametrize("bad", [dict(k_begin_host=[0, 2], k_end_host=[3, 16]), dict(k_begin_host=[10, 0], k_end_host=[16, 3]), dict(dq=A[0]),
                                 dict(dk=A[1]), dict(dv=A[1] + 128), dict(dk=A[2] - 256 * 8), dict(dq=A[9]), dict(dq=A[6]), dict(dq=A[0] + 16),
                                 dict(dq=A[0], ld_dq=264), dict(dk=A[2] - 64 * 2, ld_kv=256, ld_dkv=256)])
def test_window_gradients_with_owners(bad):
    """A key row of two sequences, and gradients over an input."""
    refused(bm.BM_ERR_INVALID_ARG, bm.window_attention_backward, *{**SIZES, **GRAD, **bad}.values())


@pytest.mark.parametrize("side", [dict(dk=A[1] + 256, dv=A[1] + 512), dict(dq=A[0] + 512, ld_q=1024, ld_dq=1024), dict(k_begin_host=[5, 10], k_end_host=[10, 16], cu_q_host=[0, 3, 5])])
def test_window_gradients_beside_inputs(side):
    """Columns of the same rows: nothing but the missing workspace is refused."""
    call = {**SIZES, **GRAD, "ld_kv": 512, "ld_dkv": 512, **side, "scratch": None}
    refused(bm.BM_ERR_WORKSPACE_TOO_SMALL, bm.window_attention_backward, *call.values())


@pytest.mark.parametrize("fn,call", [(bm.window_attention_forward, CALL), (bm.window_attention_backward, GRAD)])
@pytest.mark.parametrize("dh", [0, 12, 80, 256])
def test_window_head_sizes(fn, call, dh):
    refused(bm.BM_ERR_UNSUPPORTED, fn, *{**SIZES, **call, "dh": dh, "ld_q": 1024, "ld_kv": 512}.values())


@pytest.mark.parametrize("dtype,dh", [(0, 64), (0, 32), (1, 64)])
def test_window_workspaces(dtype, dh):
    sizes = {**SIZES, "dtype": dtype, "dh": dh}
    need = bm.window_attention_backward_scratch_bytes(*sizes.values(), 2, 5, 16)
    assert need > 0
    for bad in (dict(scratch_bytes=need - 1), dict(scratch=None)):
        refused(bm.BM_ERR_WORKSPACE_TOO_SMALL, bm.window_attention_backward, *{**sizes, **GRAD, **bad}.values())
    need = bm.window_attention_scratch_bytes(*sizes.values(), 2, 5, 16)
    if need:
        refused(bm.BM_ERR_WORKSPACE_TOO_SMALL, bm.window_attention_forward, *{**sizes, **CALL, "scratch_bytes": need - 1}.values())
    for size in (bm.window_attention_scratch_bytes, bm.window_attention_backward_scratch_bytes):
        for bad in (dict(window=0), dict(sinks=200), dict(dh=80), dict(Hq=3), dict(dtype=5)):
            assert size(*{**sizes, **bad}.values(), 2, 5, 16) == 0
        assert size(*sizes.values(), 0, 5, 16) == size(*sizes.values(), 2, -1, 16) == size(*sizes.values(), 2, 5, -1) == 0


def test_window_workspace_stays_small_for_many_short_sequences():
    """What the first keys of long sequences leave grows with the queries, not with the sequences."""
    args = (0, 1024, 4, 32, 8, 128)
    many = bm.window_attention_backward_scratch_bytes(*args, 4000, 32768, 32768)
    assert many < 4 * 32 * 32768 + 2 * 32 * 8 * 2 * 128 * 128 * 4 + (1 << 20)


@pytest.mark.parametrize("dtype,dh,Hq,Hkv", [(0, 128, 32, 8), (1, 64, 4, 4), (0, 16, 32, 1)])
def test_workspace_of_more_rows_is_enough_for_fewer(dtype, dh, Hq, Hkv):
    size = lambda S, Tq: bm.window_attention_scratch_bytes(dtype, 1024, 4, Hq, Hkv, dh, S, Tq, 100000)
    for S in (1, 64, 65, 1000):
        got = [size(S, Tq) for Tq in (0, 1, 2, 31, 64, 1000, 8192)]
        assert got == sorted(got) and size(S, 8192) <= size(S + 1, 8192) and got[1] > 0


def test_window_refuses_grids_past_32_bits():
    S = 40000
    one = np.arange(S + 1, dtype=np.int32)
    call = {**CALL, "cu_q_host": one, "k_begin_host": one[:-1], "k_end_host": one[1:], "S": S, "ld_q": 1 << 15, "ld_kv": 1 << 15}
    refused(bm.BM_ERR_INVALID_ARG, bm.window_attention_forward, *{**SIZES, "Hq": 256, "Hkv": 256, **call}.values())


def test_window_of_no_rows():
    none = np.zeros(3, np.int32)
    call = {**CALL, "cu_q_host": none, "k_begin_host": none, "k_end_host": none}
    bm.window_attention_forward(*{**SIZES, **call, "q": None, "k": None, "v": None, "o": None, "lse": None}.values(), stream=0)
    grad = {**GRAD, "cu_q_host": none, "k_begin_host": none, "k_end_host": none}
    bm.window_attention_backward(*{**SIZES, **grad, "k": None, "dk": None}.values(), stream=0)
