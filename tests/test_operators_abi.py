"""What the training operators refuse (CPU: no call here enqueues anything)."""
import math

import pytest

from paper_2609_27193_amd import layercheck as LC

A = [0x7F0000000000 + i * (1 << 34) for i in range(8)]  # never dereferenced
B, F = LC.LC_DT_BF16, LC.LC_DT_F32


def refused(fn, *args, code=LC.LC_ERR_INVALID_ARG, says="", **kw):
    with pytest.raises(LC.LCError) as e:
        fn(*args, **kw)
    assert e.value.code == code and says in str(e.value), str(e.value)


def mat(addr=A[0], rows=4, cols=8, dtype=B, stride=0, **kw):
    m = LC.matrix(addr, rows, cols, dtype, stride)
    for k, v in kw.items():
        setattr(m, k, v)
    return m


BAD_MATRICES = [(dict(addr=0), "NULL"), (dict(addr=A[0] + 1), "misaligned"), (dict(dtype=3), "dtype"), (dict(cols=0, stride=1), "columns"),
                (dict(cols=(1 << 30) + 1), "columns"), (dict(rows=(1 << 31) + 1), "rows"), (dict(stride=7), "stride"),
                (dict(stride=1 << 60), "stride"), (dict(reserved=1), "reserved")]


def bad_saved():
    for kw, says in [(dict(codes=None), "NULL"), (dict(scales=None), "NULL"), (dict(code_stride=7), "code_stride"),
                     (dict(scale_stride=0), "scale_stride"), (dict(code_stride=1 << 62), "code_stride"),
                     (dict(cols=0), "columns"), (dict(rows=(1 << 31) + 1), "rows"), (dict(rows=5), "")]:
        s = LC.saved_act(A[6], A[7], 4, 8)
        for k, v in kw.items():
            setattr(s, k, v)
        yield s, says


def embed_fwd(weight=None, tokens=A[1], dtype=LC.LC_IT_I64, n=4, out=None, **kw):
    LC.lc_embedding_forward(weight or mat(rows=10), tokens, dtype, n, out or mat(A[2]), **kw)


def embed_bwd(dout=None, tokens=A[1], dtype=LC.LC_IT_I64, n=4, dweight=None, ws=A[3], size=1 << 20, **kw):
    LC.lc_embedding_backward(dout or mat(A[2]), tokens, dtype, n, dweight or mat(rows=10), ws, size, **kw)


@pytest.mark.parametrize("kw,says", BAD_MATRICES)
def test_matrices(kw, says):
    bad = mat(**kw)
    refused(embed_fwd, weight=bad, says="weight")
    for call in (lambda: embed_fwd(out=bad), lambda: embed_bwd(dout=bad), lambda: embed_bwd(dweight=bad),
                 lambda: LC.lc_norm_forward(norm(), bad, mat(A[2])), lambda: LC.lc_norm_forward(norm(), mat(A[2]), bad),
                 lambda: LC.lc_act_save(bad, LC.saved_act(A[6], A[7], 4, 8)),
                 lambda: LC.lc_act_load(LC.saved_act(A[6], A[7], 4, 8), bad), lambda: norm_bwd(dy=bad),
                 lambda: norm_bwd(x=bad, mean=A[5]), lambda: norm_bwd(dx=bad), lambda: wgrad(dy=bad), lambda: wgrad(dweight=bad)):
        refused(call, says=says)


def test_embedding():
    refused(embed_fwd, tokens=0, says="NULL")
    refused(embed_fwd, tokens=A[1] + 4, says="misaligned")
    refused(embed_fwd, tokens=A[1] + 2, dtype=LC.LC_IT_I32, says="misaligned")
    refused(embed_fwd, dtype=3, says="token dtype")
    refused(embed_fwd, out=mat(A[2], rows=3), says="out is 3 x 8, not 4 x 8")
    refused(embed_fwd, out=mat(A[2], cols=9), says="out")
    refused(embed_fwd, out=mat(A[0] + 16), says="overlap")
    refused(embed_fwd, out=mat(A[1]), says="overlap")
    many = dict(n=5000, dout=mat(A[2], rows=5000))  # sorted in the workspace
    refused(embed_bwd, ws=0, says="workspace is NULL", **many)
    refused(embed_bwd, ws=A[3] + 8, says="aligned", **many)
    refused(embed_bwd, size=100, code=LC.LC_ERR_CAPACITY, says="workspace", **many)
    refused(embed_bwd, ws=A[2], says="overlap", **many)
    refused(embed_bwd, dout=mat(A[2], cols=9), says="dout")
    refused(embed_bwd, dweight=mat(A[2], rows=10), says="overlap")
    lib = LC.load_library()
    assert lib.lc_embedding_backward(mat(A[2]), A[1], 2, 4, 0, 1.0, 2, mat(rows=10), A[3], 1 << 20, None) == LC.LC_ERR_INVALID_ARG
    assert lib.lc_embedding_forward(None, A[1], 2, 4, 0, 1.0, mat(), None) == LC.LC_ERR_INVALID_ARG
    assert LC.lc_embedding_backward_workspace(1 << 40, 8) == 0
    assert LC.lc_embedding_backward_workspace(0, 8) == 0
    assert LC.lc_embedding_backward_workspace(5000, 8) >= 5000 * 8


def norm(kind=LC.LC_NORM_LAYER, weight=A[4], bias=A[5], dtype=F, eps=1e-5):
    return LC.norm_params(kind, weight, bias, dtype, eps)


def norm_bwd(params=None, dy=None, rstd=A[4], dx=None, dweight=A[3], dbias=0, dtype=F, ws=A[2], size=1 << 20, x=None, **kw):
    if x is None and "saved" not in kw:
        x, kw = mat(A[1]), {"mean": A[5], **kw}
    LC.lc_norm_backward(params or norm(weight=0, bias=0), dy or mat(), rstd, dx, dweight, dbias, dtype, ws, size, x=x, **kw)


def test_norms():
    fwd = lambda p, x=None, y=None, **kw: LC.lc_norm_forward(p, x or mat(), y or mat(A[1]), **kw)  # noqa: E731
    refused(fwd, norm(kind=2), says="kind")
    refused(fwd, norm(dtype=0), says="param dtype")
    refused(fwd, norm(eps=-1e-9), says="eps")
    refused(fwd, norm(eps=math.nan), says="eps")
    refused(fwd, norm(eps=math.inf), says="eps")
    refused(fwd, norm(weight=A[4] + 2), says="misaligned")
    refused(fwd, norm(bias=A[4] + 2), says="misaligned")
    refused(fwd, norm(kind=LC.LC_NORM_RMS), says="no bias")
    refused(fwd, norm(kind=LC.LC_NORM_RMS, bias=0), mean=A[2], says="no mean")
    refused(fwd, norm(), y=mat(A[1], dtype=F), says="dtype")
    refused(fwd, norm(), y=mat(A[1], rows=5), says="y is")
    refused(fwd, norm(), mean=A[2] + 1, says="mean")
    refused(fwd, norm(), rstd=A[2] + 2, says="rstd")
    refused(fwd, norm(), y=mat(), says="overlap")
    refused(fwd, norm(), rstd=A[1], says="overlap")
    refused(fwd, norm(), mean=A[2], rstd=A[2] + 8, says="overlap")
    for s, says in bad_saved():
        refused(fwd, norm(), saved=s, says=says)
    both = LC.saved_act(A[0], A[7], 4, 8)
    refused(norm_bwd, x=mat(A[1]), mean=A[5], saved=both, says="exactly one")
    lib = LC.load_library()
    assert lib.lc_norm_backward(norm(), mat(), None, None, A[4], None, None, None, None, F, 0, None, 0, None) == LC.LC_ERR_INVALID_ARG
    refused(norm_bwd, x=mat(A[1]), says="mean or rstd")
    refused(norm_bwd, rstd=0, says="mean or rstd")
    refused(norm_bwd, saved=LC.saved_act(A[1], A[7], 4, 8), mean=A[5], says="mean goes with")
    refused(norm_bwd, params=norm(LC.LC_NORM_RMS, 0, 0), x=mat(A[1]), mean=A[5], says="mean goes with")
    refused(norm_bwd, params=norm(LC.LC_NORM_RMS, 0, 0), x=mat(A[1]), dbias=A[6], says="no bias")
    refused(norm_bwd, x=mat(A[1], dtype=F), mean=A[5], says="dtype")
    refused(norm_bwd, x=mat(A[1], rows=5), mean=A[5], says="x is")
    refused(norm_bwd, dx=mat(A[6], cols=7), says="dx is")
    refused(norm_bwd, dx=mat(A[6], dtype=F), says="dtype")
    refused(norm_bwd, dx=mat(A[1]), says="overlap")
    refused(norm_bwd, dweight=A[3] + 2, says="misaligned")
    refused(norm_bwd, dbias=A[3] + 4, says="overlap")
    refused(norm_bwd, dtype=7, says="gradient dtype")
    refused(norm_bwd, ws=0, says="workspace is NULL")
    refused(norm_bwd, size=16, code=LC.LC_ERR_CAPACITY)
    refused(norm_bwd, ws=A[3], says="overlap")
    for s, says in bad_saved():
        refused(norm_bwd, saved=s, says=says)
    assert LC.lc_norm_backward_workspace(1, 1 << 31) == 0


def wgrad(dy=None, saved=None, dweight=None, ws=A[2], size=1 << 20, **kw):
    LC.lc_linear_wgrad(dy or mat(cols=6), saved or LC.saved_act(A[6], A[7], 4, 8), dweight or mat(A[1], 6, 8), ws, size, **kw)


def test_saved_activations_and_wgrad():
    for s, says in bad_saved():
        refused(LC.lc_act_save, mat(), s, says=says)
        refused(LC.lc_act_load, s, mat(), says=says)
        refused(wgrad, saved=s, says=says)
    refused(LC.lc_act_save, mat(), LC.saved_act(A[0], A[7], 4, 8), says="overlap")
    refused(LC.lc_act_save, mat(), LC.saved_act(A[6], A[6] + 31, 4, 8), says="overlap")
    refused(LC.lc_act_load, LC.saved_act(A[6], A[0], 4, 8), mat(), says="overlap")
    refused(wgrad, dweight=mat(A[1], 5, 8), says="dweight is 5 x 8, not 6 x 8")
    refused(wgrad, dweight=mat(A[1], 6, 9), says="dweight")
    refused(wgrad, dweight=mat(A[0], 6, 8), says="overlap")
    refused(wgrad, col_scale=A[4], param_dtype=5, says="param dtype")
    refused(wgrad, col_scale=A[4] + 2, says="misaligned")
    refused(wgrad, col_shift=A[4] + 1, param_dtype=B, says="misaligned")
    refused(wgrad, dbias=A[4] + 1, says="misaligned")
    refused(wgrad, dbias=A[1], says="overlap")
    rows = 1 << 14  # split over the tokens: a workspace is needed
    big = dict(dy=mat(rows=rows, cols=64), saved=LC.saved_act(A[6], A[7], rows, 64), dweight=mat(A[1], 64, 64))
    assert LC.lc_linear_wgrad_workspace(rows, 64, 64) > 0
    refused(wgrad, ws=0, says="workspace is NULL", **big)
    refused(wgrad, size=64, code=LC.LC_ERR_CAPACITY, **big)
    refused(wgrad, ws=A[0], size=1 << 30, says="overlap", **big)
    assert LC.lc_linear_wgrad_workspace(1, 0, 5) == 0 and LC.lc_linear_wgrad_workspace(1, 5, 1 << 31) == 0
    assert LC.lc_linear_wgrad_workspace(1, 1 << 30, 1 << 30) == 0


def test_columns_beside_each_other_are_apart():
    """Two column ranges of one buffer share no byte, however their rows interleave; one column more, and they do."""
    buf = A[0]
    left, right = mat(buf, cols=8, stride=16), mat(buf + 16, cols=8, stride=16)
    wide = mat(buf, cols=9, stride=16)
    refused(LC.lc_norm_forward, norm(), left, right, mean=A[2], rstd=A[2], says="mean and rstd")  # y and x passed
    refused(LC.lc_norm_forward, norm(), wide, LC.matrix(buf + 16, 4, 9, B, 16), mean=A[2], rstd=A[2], says="y and x")


def test_nothing_to_do_is_no_error():
    """No rows and no tokens: done before anything is asked of the GPU."""
    e = lambda cols=8: LC.matrix(0, 0, cols, B)  # noqa: E731
    LC.lc_embedding_forward(mat(rows=10), 0, LC.LC_IT_I64, 0, e())
    LC.lc_act_save(e(), LC.saved_act(0, 0, 0, 8))
    LC.lc_act_load(LC.saved_act(0, 0, 0, 8), e())
    LC.lc_norm_forward(norm(), e(), e())
    LC.lc_embedding_backward(mat(A[2], 4), A[1], LC.LC_IT_I64, 4, LC.matrix(0, 0, 8, B), A[3], 1 << 20)
