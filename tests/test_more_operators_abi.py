"""What the residual norm and the orthogonalised update refuse (CPU: no call here enqueues anything)."""
import math

import pytest

from paper_2609_27193_amd import layercheck as LC
from tests.test_operators_abi import A, BAD_MATRICES, bad_saved, mat, refused

B, F = LC.LC_DT_BF16, LC.LC_DT_F32
FAR = [A[0] + 8 * (1 << 34) + i * (1 << 34) for i in range(16)]  # never dereferenced


def params(kind=LC.LC_NORM_RMS, weight=A[5], bias=0, dtype=B, eps=1e-5):
    return LC.norm_params(kind, weight, bias, dtype, eps)


def saved(i=0, rows=4, cols=8):
    return LC.saved_act(FAR[2 * i], FAR[2 * i + 1], rows, cols)


def forward(prm=None, x=None, residual=None, h=..., y=..., **kw):
    LC.lc_residual_norm_forward(prm or params(), x or mat(), residual or mat(A[1]), mat(A[2]) if h is ... else h,
                                mat(A[3]) if y is ... else y, **kw)


def backward(prm=None, dy=None, dh=None, rstd=A[2], dx=..., dresidual=None, dweight=A[4], dbias=None, grad=F, ws=A[6], size=1 << 24,
             h=..., **kw):
    LC.lc_residual_norm_backward(prm or params(), dy or mat(), dh or mat(A[1]), rstd, mat(A[3]) if dx is ... else dx, dresidual, dweight,
                                 dbias, grad, ws, size, h=mat(A[7]) if h is ... else h, **kw)


@pytest.mark.parametrize("kw,says", BAD_MATRICES)
@pytest.mark.parametrize("name", ["x", "residual", "h", "y"])
def test_forward_matrices(name, kw, says):
    refused(forward, **{name: mat(**kw)}, says=says)


@pytest.mark.parametrize("kw,says", BAD_MATRICES)
@pytest.mark.parametrize("name", ["dy", "dh", "dx", "dresidual", "h"])
def test_backward_matrices(name, kw, says):
    refused(backward, **{name: mat(**kw)}, says=says)


def test_forward():
    for name in ("residual", "h", "y"):
        refused(forward, **{name: mat(FAR[3], rows=5)}, says=name)
        refused(forward, **{name: mat(FAR[3], cols=9, stride=9)}, says=name)
    refused(forward, y=mat(A[3], dtype=F), says="dtype")
    refused(forward, h=mat(A[2], dtype=F), says="dtype")
    refused(forward, x=mat(dtype=F), y=mat(A[3], dtype=F), says="residual")  # a bf16 stream beside fp32 layers
    refused(forward, y=None, says="y or y_saved")
    refused(forward, prm=params(bias=A[6]), says="bias")
    refused(forward, mean=A[6], says="mean")
    refused(forward, rstd=A[6] + 2, says="misaligned")
    refused(forward, prm=params(kind=LC.LC_NORM_LAYER), mean=A[6] + 1, says="misaligned")
    for eps in (-1.0, math.nan, math.inf):
        refused(forward, prm=params(eps=eps), says="eps")
    for bad, says in bad_saved():
        refused(forward, saved=bad, says=says)
        refused(forward, y_saved=bad, says=says)
    lib = LC.load_library()
    assert lib.lc_residual_norm_forward(None, mat(), mat(A[1]), None, mat(A[3]), None, None, None, None, None) == LC.LC_ERR_INVALID_ARG
    for i in range(2):
        args = [mat(), mat(A[1])]
        args[i] = None
        assert lib.lc_residual_norm_forward(params(), *args, None, mat(A[3]), None, None, None, None, None) == LC.LC_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(h=mat(A[1])), dict(h=mat(A[0])), dict(y=mat(A[0] + 16)), dict(y=mat(A[2])), dict(rstd=A[1]),
                                dict(y_saved=LC.saved_act(A[0] + 8, FAR[0], 4, 8)), dict(saved=saved(1), y_saved=saved(1)),
                                dict(y_saved=LC.saved_act(FAR[0], A[2], 4, 8)), dict(h=mat(A[5]))])
def test_forward_overlaps(kw):
    refused(forward, says="overlap", **kw)


def test_backward():
    for name in ("dh", "dx", "dresidual", "h"):
        refused(backward, **{name: mat(FAR[3], rows=5)}, says=name)
    refused(backward, dx=mat(A[3], dtype=F), says="dx")
    refused(backward, dresidual=mat(FAR[0], dtype=F), says="dresidual")
    refused(backward, h=mat(A[7], dtype=F), says="h has")
    refused(backward, dy=mat(dtype=F), dx=mat(A[3], dtype=F), says="residual")
    refused(backward, h=None, says="exactly one")
    refused(backward, saved=saved(), says="exactly one")
    refused(backward, rstd=0, says="rstd")
    refused(backward, rstd=A[2] + 2, says="misaligned")
    refused(backward, mean=FAR[0], says="mean")
    refused(backward, prm=params(kind=LC.LC_NORM_LAYER), says="mean")
    refused(backward, prm=params(kind=LC.LC_NORM_LAYER), h=None, saved=saved(), mean=FAR[8], says="mean")
    refused(backward, dbias=FAR[0], says="bias")
    refused(backward, grad=7, says="dtype")
    refused(backward, dweight=A[4] + 2, says="misaligned")
    refused(backward, accumulate=2, says="accumulate")
    refused(backward, ws=0, says="workspace")
    refused(backward, ws=A[6] + 8, says="aligned")
    refused(backward, size=LC.lc_norm_backward_workspace(4, 8) - 1, says="workspace", code=LC.LC_ERR_CAPACITY)
    for bad, says in bad_saved():
        refused(backward, h=None, saved=bad, says=says)
    lib = LC.load_library()
    assert lib.lc_residual_norm_backward(params(), mat(), None, mat(A[7]), None, A[2], None, mat(A[3]), None, None, None, F, 0, None, 0,
                                         None) == LC.LC_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(dx=mat(A[0])), dict(dx=mat(A[1])), dict(dx=mat(A[7] + 16)), dict(dresidual=mat(A[3])), dict(ws=A[3]),
                                dict(dweight=A[1]), dict(dresidual=mat(A[1])), dict(dweight=A[6])])
def test_backward_overlaps(kw):
    refused(backward, says="overlap", **kw)


# ---- the orthogonalised update ---------------------------------------------------------------------------------------------


def ortho(prm=None, grads=None, out=None, momenta=None, ws=FAR[15], size=1 << 33, n=2):
    LC.lc_orthogonalize(prm or LC.orthogonalize_params(5), grads or [mat(A[i]) for i in range(n)],
                        out or [mat(FAR[i]) for i in range(n)], ws, size, momenta=momenta)


@pytest.mark.parametrize("kw,says", BAD_MATRICES)
@pytest.mark.parametrize("name,at", [("grads", 0), ("grads", 1), ("out", 0), ("out", 1), ("momenta", 1)])
def test_ortho_matrices(name, at, kw, says):
    first = {"grads": A[0], "out": FAR[0], "momenta": FAR[4]}[name]
    ms = [mat(first + i * (1 << 34), dtype=F if name == "momenta" else B) for i in range(2)]
    ms[at] = mat(**{"addr": first + at * (1 << 34), **({"dtype": F} if name == "momenta" else {}), **kw})
    if kw.get("addr") == A[0] + 1 and name == "momenta":
        ms[at].data = first + 1
    refused(ortho, **{name: ms}, says=says)


def test_ortho_params():
    P = LC.orthogonalize_params
    for bad, says in [(P(0, None), "steps"), (P(33, None), "steps"), (P(5, momentum=1.0), "momentum"), (P(5, momentum=-0.1), "momentum"),
                      (P(5, momentum=math.nan), "momentum"), (P(5, eps=-1.0), "eps"), (P(5, eps=math.inf), "eps"),
                      (P(5, scale=math.nan), "scale"), (P(5, scale=2.0 ** 65), "scale"), (P(5, scale=-(2.0 ** -65)), "scale"), (P(5, scale=math.inf), "scale"), (P(5, (1, math.nan, 0)), "coefs"),
                      (P(5, (1, math.inf, 0)), "coefs"), (P(5, (40.0, 0, 0)), "singular"), (P(5, (2.0 ** -7, 0, 0)), "singular"),
                      (P(3, [(1, 0, 0), (1, 0, 0), (1, 2e9, 0)]), "singular")]:
        refused(ortho, prm=bad, says=says)
    flag = P(5)
    flag.nesterov = 2
    refused(ortho, prm=flag, says="nesterov")
    lib = LC.load_library()
    two = LC.lc_matrix * 2
    g, o = two(mat(A[0]), mat(A[1])), two(mat(FAR[0]), mat(FAR[1]))
    assert lib.lc_orthogonalize(None, 2, g, None, o, FAR[15], 1 << 33, None) == LC.LC_ERR_INVALID_ARG
    assert lib.lc_orthogonalize(P(5), 2, None, None, o, FAR[15], 1 << 33, None) == LC.LC_ERR_INVALID_ARG
    assert lib.lc_orthogonalize(P(5), 2, g, None, None, FAR[15], 1 << 33, None) == LC.LC_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        P(5, [(1, 0, 0)] * 4)
    with pytest.raises(ValueError):
        LC.lc_orthogonalize(P(5), [mat()], [], 0, 0)


def test_ortho_shapes_and_types():
    refused(ortho, grads=[mat(A[0]), mat(A[1], rows=5)], says="grads")
    refused(ortho, out=[mat(FAR[0]), mat(FAR[1], cols=9, stride=9)], says="out")
    refused(ortho, grads=[mat(A[0]), mat(A[1], dtype=F)], says="dtypes")
    refused(ortho, out=[mat(FAR[0], dtype=F), mat(FAR[1])], says="dtypes")
    refused(ortho, momenta=[mat(FAR[4]), mat(FAR[5])], says="LC_DT_F32")  # a momentum is kept in 32 bits
    refused(ortho, n=65, grads=[mat(A[0])] * 65, out=[mat(FAR[0])] * 65, says="at most 64")
    for shape in (dict(rows=65537), dict(cols=65537, stride=65537)):
        refused(ortho, grads=[mat(A[0], **shape)], out=[mat(FAR[0], **shape)], says="65536")


def test_ortho_workspace():
    need = LC.lc_orthogonalize_workspace(2, 4, 8, B)
    assert need > 0 and need % 16 == 0
    assert LC.lc_orthogonalize_workspace(2, 4, 8, F) == need  # few rows: two planes for either result
    assert LC.lc_orthogonalize_workspace(2, 400, 800, F) > LC.lc_orthogonalize_workspace(2, 400, 800, B)
    for bad in [(0, 4, 8, B), (65, 4, 8, B), (2, 0, 8, B), (2, 4, 0, B), (2, 65537, 8, B), (2, 4, 65537, B), (2, 4, 8, 3)]:
        assert LC.lc_orthogonalize_workspace(*bad) == 0
    assert LC.lc_orthogonalize_workspace(3, 700, 90, F) == LC.lc_orthogonalize_workspace(3, 90, 700, F)
    refused(ortho, size=need - 1, says="workspace", code=LC.LC_ERR_CAPACITY)
    refused(ortho, ws=0, says="workspace")
    refused(ortho, ws=FAR[15] + 8, says="aligned")


@pytest.mark.parametrize("kw", [dict(out=[mat(A[0]), mat(FAR[1])]), dict(out=[mat(FAR[0]), mat(FAR[0])]), dict(out=[mat(A[1] + 32), mat(FAR[1])]),
                                dict(ws=A[0]), dict(ws=FAR[1]), dict(ws=FAR[0] - 1024),
                                dict(momenta=[mat(FAR[4], dtype=F), mat(FAR[4], dtype=F)]), dict(momenta=[mat(A[1], dtype=F), mat(FAR[4], dtype=F)])])
def test_ortho_overlaps(kw):
    refused(ortho, says="overlap", **kw)


def test_ortho_same_gradient_twice_is_no_overlap():
    """What is only read may be given twice; the call gets as far as the workspace."""
    refused(ortho, grads=[mat(A[0]), mat(A[0])], size=0, says="workspace", code=LC.LC_ERR_CAPACITY)
    refused(ortho, grads=[mat(A[0]), mat(A[0])], out=[mat(FAR[0]), mat(FAR[0] + 16)], says="overlap")


def test_the_mixed_step_needs_a_context():
    lib = LC.load_library()
    prm = LC.lc_muon_params(LC.lc_adamw_params(1e-3, 0.9, 0.95, 1e-8, 0, 1), 1e-3, 0)
    assert lib.lc_muon_step_score(None, 1, None, B, None, None, prm) == LC.LC_ERR_INVALID_ARG
