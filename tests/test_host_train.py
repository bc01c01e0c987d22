"""What the operators of a training step refuse, before anything is launched (no GPU)."""
import pytest

from paper_2605_25451_amd import binding as bm

P, Q, R, S, W = 4096, 8192, 12288, 16384, 20480              # addresses that are never followed


def refused(status, fn, *args):
    with pytest.raises(bm.BmError) as e:
        fn(*args, stream=0)
    assert e.value.status == status and bm.last_error()


LOOKUP = dict(dtype=0, V=100, d=16, table=P, ld_table=16, ids=Q, T=4, scale=1.0, y=R, ld_y=16)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(V=0), dict(d=0), dict(T=-1), dict(ld_table=15), dict(ld_y=8),
                                 dict(table=None), dict(ids=None), dict(y=None), dict(table=P + 2), dict(y=R + 8),
                                 dict(ids=Q + 4), dict(d=(1 << 30) + 1, ld_table=(1 << 30) + 1, ld_y=(1 << 30) + 1), dict(T=1 << 30, d=8192, ld_table=8192, ld_y=8192)])
def test_lookup_refusals(bad):
    refused(bm.BM_ERR_INVALID_ARG, bm.embedding_forward, *{**LOOKUP, **bad}.values())


GRAD = dict(dtype=0, V=100, d=16, dy=P, ld_dy=16, ids=Q, T=40, scale=1.0, dtable=R, ld_dtable=16, scratch=S,
            scratch_bytes=1 << 30)


@pytest.mark.parametrize("bad", [dict(dtype=-1), dict(V=-3), dict(d=0), dict(T=-1), dict(ld_dy=15), dict(ld_dtable=15),
                                 dict(dy=None), dict(ids=None), dict(dtable=None), dict(dy=P + 2), dict(dtable=R + 4),
                                 dict(scratch=S + 8), dict(T=(1 << 30) + 1)])
def test_embedding_gradient_refusals(bad):
    refused(bm.BM_ERR_INVALID_ARG, bm.embedding_backward, *{**GRAD, **bad}.values())


@pytest.mark.parametrize("bad", [dict(scratch_bytes=bm.embedding_backward_scratch_bytes(40, 16) - 1), dict(scratch=None),
                                 dict(scratch_bytes=0)])
def test_embedding_gradient_workspace(bad):
    refused(bm.BM_ERR_WORKSPACE_TOO_SMALL, bm.embedding_backward, *{**GRAD, **bad}.values())


def test_embedding_workspace_grows_with_tokens_and_columns():
    sizes = [bm.embedding_backward_scratch_bytes(T, 64) for T in (1, 2, 777, 2048, 2049, 8192, 8193, 32768, 32769, 1 << 20)]
    assert all(b > 0 for b in sizes)
    assert all(b >= a for a, b in zip(sizes, sizes[1:]))
    assert bm.embedding_backward_scratch_bytes(777, 65) >= bm.embedding_backward_scratch_bytes(777, 64)
    for T, d in ((0, 8), (8, 0), (-1, 8), ((1 << 30) + 1, 8), (8, (1 << 30) + 1)):
        assert bm.embedding_backward_scratch_bytes(T, d) == 0


LOSS = dict(dtype=0, T=4, V=100, logits=P, ld=104, labels=Q, weight=None, loss=R, dlogits=S, ld_d=104, scratch=W,
            scratch_bytes=1 << 30)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(T=-1), dict(V=0), dict(ld=99), dict(ld_d=99), dict(logits=None),
                                 dict(labels=None), dict(loss=None, dlogits=None), dict(logits=P + 2), dict(labels=Q + 4),
                                 dict(weight=W + 4), dict(loss=R + 4), dict(dlogits=S + 2), dict(scratch=W + 8),
                                 dict(dlogits=P, ld_d=112), dict(V=(1 << 31) - 1, ld=(1 << 31) - 1, ld_d=(1 << 31) - 1)])
def test_cross_entropy_refusals(bad):
    refused(bm.BM_ERR_INVALID_ARG, bm.cross_entropy, *{**LOSS, **bad}.values())


def test_cross_entropy_workspace():
    need = bm.cross_entropy_scratch_bytes(0, 4, 100)
    if need:
        refused(bm.BM_ERR_WORKSPACE_TOO_SMALL, bm.cross_entropy, *{**LOSS, "scratch_bytes": need - 1}.values())
        refused(bm.BM_ERR_WORKSPACE_TOO_SMALL, bm.cross_entropy, *{**LOSS, "scratch": None}.values())
    for args in ((2, 4, 100), (0, 0, 100), (0, 4, 0)):
        assert bm.cross_entropy_scratch_bytes(*args) == 0


def test_no_tokens_is_nothing_to_do():
    bm.embedding_forward(0, 100, 16, None, 16, None, 0, 1.0, None, 16, stream=0)
    bm.embedding_backward(0, 100, 16, None, 16, None, 0, 1.0, None, 16, None, 0, stream=0)
    bm.cross_entropy(0, 0, 100, None, 100, None, None, None, None, 100, stream=0)


ORTHO = dict(dtype=0, batch=3, M=20, N=30, grad=P, ld_g=30, stride_g=600, out=Q, ld_o=30, stride_o=600,
             coefficients=(3.4445, -4.7750, 2.0315), steps=5, eps=1e-7, scratch=R, scratch_bytes=1 << 30)


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(batch=-1), dict(M=0), dict(N=-1), dict(ld_g=29), dict(ld_o=29),
                                 dict(stride_g=-1), dict(stride_o=-600), dict(stride_o=599), dict(stride_o=30, ld_o=89),
                                 dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")),
                                 dict(coefficients=None), dict(grad=None), dict(out=None), dict(grad=P + 4), dict(out=Q + 2),
                                 dict(scratch=R + 8), dict(M=(1 << 20) + 1), dict(M=1 << 20, N=1 << 20, ld_g=1 << 20, ld_o=1 << 20)])
def test_orthogonalize_refusals(bad):
    refused(bm.BM_ERR_INVALID_ARG, bm.orthogonalize, *{**ORTHO, **bad}.values())


@pytest.mark.parametrize("c", [(9.0, 0.0, 0.0), (1.6, 0.0, 0.0), (float("nan"), 0.0, 0.0), (1.0, float("inf"), 0.0), (3.0, 4.0, 5.0)])
def test_orthogonalize_refuses_coefficients_that_diverge(c):
    refused(bm.BM_ERR_UNSUPPORTED, bm.orthogonalize, *{**ORTHO, "coefficients": c}.values())


def test_orthogonalize_workspace():
    for dtype in (0, 1):
        need = bm.orthogonalize_scratch_bytes(dtype, 3, 20, 30)
        assert need > 0
        for bad in (dict(scratch_bytes=need - 1), dict(scratch=None)):
            refused(bm.BM_ERR_WORKSPACE_TOO_SMALL, bm.orthogonalize, *{**ORTHO, "dtype": dtype, **bad}.values())
    for args in ((2, 1, 8, 8), (0, 0, 8, 8), (0, 1, 0, 8), (0, 1, 8, (1 << 20) + 1), (0, 1, 1 << 20, 1 << 20)):
        assert bm.orthogonalize_scratch_bytes(*args) == 0
    bm.orthogonalize(0, 0, 8, 8, None, 8, 64, None, 8, 64, (1.0, 0.0, 0.0), 1, 0.0, None, 0, stream=0)


@pytest.mark.parametrize("dtype,batch,ld_g,stride_g,out,ld_o,stride_o", [
    (0, 2, 30, 600, 0, 30, 600), (0, 1, 30, 600, 0, 30, 600), (1, 2, 30, 0, 0, 30, 600), (1, 2, 32, 640, 0, 30, 600),
    (1, 2, 30, 640, 0, 30, 600), (1, 2, 30, 600, 16, 30, 600), (0, 2, 30, 600, -16, 30, 600), (1, 2, 30, 600, 4784, 30, 600)])
def test_orthogonalize_refuses_results_that_overlap_the_gradient(dtype, batch, ld_g, stride_g, out, ld_o, stride_o):
    refused(bm.BM_ERR_INVALID_ARG, bm.orthogonalize, dtype, batch, 20, 30, 1 << 20, ld_g, stride_g, (1 << 20) + out, ld_o, stride_o,
            (1.0, 0.0, 0.0), 1, 0.0, 1 << 30, 1 << 30)
    assert "overlaps" in bm.last_error()
