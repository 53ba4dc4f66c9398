"""The training operators' rows where their sizes are even and their addresses are not, mixed types, and more rows than
their blocks take in three turns.

As in the other tests of them, a bound is U32 = 2^-24 for each fp32 rounding that an addend passes through, and the rounding of
the result's type.  A row's sum passes a thread's own elements (24 at most), six steps within a wave and up to 16 waves; a dozen
roundings are the formula's own."""
import math

import pytest
import torch

from paper_2609_27193_amd import layercheck as LC
from tests.test_operators_gpu import DT, U32, Guarded, Kept, close, gen, kept_normal, norm_reference, space, stream

pytestmark = pytest.mark.gpu

ROW = 24 + 6 + 16 + 12


def over_rows(rows):
    # 256 blocks at least take turns at the rows, four side by side at most; 1280 parts at most in 32 slices, then the slices
    return rows // 256 + 1 + 4 + 40 + 32


NORM = [(3, 64), (2, 512), (5, 1024), (3, 2048), (2, 4096), (3, 5120), (2, 8192), (3, 16384),  # whole groups, odd places
        (17000, 64), (9000, 520), (6500, 2048), (4100, 4096), (1700, 8192), (900, 16384)]       # more than three turns
PLACES = [(1, 1), (8, 3)]


def norm_case(rows, dim, dtype, param, pad, off, rms, weighted=True):
    dt, pt = DT[dtype][0], DT[param][0]
    g = gen(rows + 13 * dim)
    x = Guarded(rows, dim, dt, pad, off, torch.randn(rows, dim, generator=g, device="cuda") * 2 + 0.5)
    w = Guarded(1, dim, pt, 0, off, 1 + 0.3 * torch.randn(1, dim, generator=g, device="cuda"))
    b = Guarded(1, dim, pt, 0, off, 0.3 * torch.randn(1, dim, generator=g, device="cuda"))
    prm = LC.norm_params(LC.LC_NORM_RMS if rms else LC.LC_NORM_LAYER, w.addr if weighted else 0,
                         0 if rms or not weighted else b.addr, DT[param][1], 1e-5)
    w64 = w.view.double()[0] if weighted else torch.ones(dim, dtype=torch.float64, device="cuda")
    b64 = b.view.double()[0] if weighted and not rms else torch.zeros(dim, dtype=torch.float64, device="cuda")
    return g, x, prm, w64, b64, (w, b)


@pytest.mark.parametrize("rows,dim", NORM)
@pytest.mark.parametrize("dtype,param,pad,off", [("bf16", "f32", 1, 1), ("f32", "bf16", 8, 3)])
@pytest.mark.parametrize("rms", [False, True])
def test_norm(rows, dim, dtype, param, pad, off, rms):
    dt, _, u = DT[dtype]
    _, x, prm, w, b, held = norm_case(rows, dim, dtype, param, pad, off, rms)
    y, k = Guarded(rows, dim, dt, pad, off), Kept(rows, dim, pad=pad, off=off)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    LC.lc_norm_forward(prm, x.matrix(), y.matrix(), 0 if rms else mean.data_ptr(), rstd.data_ptr(), k.act, stream())
    rm, rr, rn, ry = norm_reference(x.view, w, b, rms, 1e-5)
    size = x.view.double().abs().mean(1, keepdim=True)
    shift = ROW * U32 * size * (0 if rms else 1)
    if not rms:
        close(mean, rm[:, 0], ROW * U32 * size[:, 0])
    close(rstd, rr[:, 0], (ROW * U32 * rr + shift ** 2 * rr ** 3)[:, 0])
    n_tol = ROW * U32 * rn.abs() + shift * rr + 2 * U32 * rm.abs() * rr
    close(y.view, ry, 2 * u * ry.abs() + n_tol * w.abs() + 4 * U32 * (ry.abs() + b.abs()))
    step = torch.ldexp(torch.ones_like(rn), (k.scales.view.long() - 127 - 10).repeat_interleave(32, 1)[:, :dim])
    close(k.values(), rn, torch.maximum(rn.abs() / 16, step) * (1 + 1e-6) + 2 * n_tol)
    assert y.intact() and k.intact() and x.intact()


@pytest.mark.parametrize("rows,dim", NORM)
@pytest.mark.parametrize("rms,source,dtype,param,grad", [(False, "x", "bf16", "f32", "bf16"), (False, "x", "f32", None, "f32"),
                                                         (False, "kept", "f32", "bf16", "bf16"), (False, "kept", "bf16", "f32", "f32"),
                                                         (True, "x", "f32", "bf16", "f32"), (True, "kept", "bf16", None, "f32")])
def test_norm_gradient(rows, dim, dtype, param, grad, source, rms):
    """`param` None: no weight."""
    pad, off = PLACES[source == "kept"]
    dt, _, u = DT[dtype]
    gt, gcode, u_grad = DT[grad]
    g, x, prm, w, _, held = norm_case(rows, dim, dtype, param or "f32", pad, off, rms, param is not None)
    dy = Guarded(rows, dim, dt, pad, off, torch.randn(rows, dim, generator=g, device="cuda"))
    rstd = torch.rand(rows, generator=g, device="cuda") + 0.5
    mean = torch.randn(rows, generator=g, device="cuda")
    rs, k = rstd[:, None].double(), None
    if source == "x":
        m = mean[:, None].double() * (0 if rms else 1)
        n = (x.view.double() - m) * rs
        n_tol = 3 * U32 * (n.abs() + m.abs() * rs)
    else:
        k = kept_normal(rows, dim, dim, pad, off)
        n, n_tol = k.values(), torch.zeros(1, 1, dtype=torch.float64, device="cuda").expand(rows, dim)
    d = dy.view.double()
    gw = d * w
    c1 = gw.mean(1, keepdim=True) * (0 if rms else 1)
    c2 = (gw * n).mean(1, keepdim=True)
    rdx = rs * (gw - c1 - n * c2)
    c1_tol = ROW * U32 * gw.abs().mean(1, keepdim=True) * (0 if rms else 1)
    c2_tol = ROW * U32 * (gw * n).abs().mean(1, keepdim=True) + (gw.abs() * n_tol).mean(1, keepdim=True)
    dx_tol = rs * (4 * U32 * (gw.abs() + c1.abs() + (n * c2).abs()) + c1_tol + n.abs() * c2_tol + n_tol * c2.abs())
    need = LC.lc_norm_backward_workspace(rows, dim)
    buf, ws, _ = space(need)
    dx = Guarded(rows, dim, dt, pad, off)
    dw, db = (Guarded(1, dim, gt, 0, off, torch.full((1, dim), math.nan, device="cuda")) for _ in "wb")
    LC.lc_norm_backward(prm, dy.matrix(), rstd.data_ptr(), dx.matrix(), dw.addr, 0 if rms else db.addr, gcode, ws, need,
                        x=x.matrix() if k is None else None, mean=mean.data_ptr() if k is None and not rms else 0,
                        saved=k.act if k else None, stream=stream())
    close(dx.view, rdx, 2 * u * rdx.abs() + dx_tol)
    deep = over_rows(rows)
    want, size = (d * n).sum(0), (d * n).abs().sum(0)
    close(dw.view[0], want, 2 * u_grad * want.abs() + deep * U32 * size * (1 + u_grad) + (d.abs() * n_tol).sum(0))
    if not rms:
        want = d.sum(0)
        close(db.view[0], want, 2 * u_grad * want.abs() + deep * U32 * d.abs().sum(0) * (1 + u_grad))
    assert bool((buf[need:] == 0xA5).all())
    assert dx.intact() and dw.intact() and db.intact() and dy.intact() and x.intact()


@pytest.mark.parametrize("n,vocab,dim", [(300, 900, 64), (2000, 50, 520), (3000, 400, 2048), (6000, 3000, 136), (20000, 700, 256)])
@pytest.mark.parametrize("w,o", [("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("pad,off", PLACES)
def test_embedding(n, vocab, dim, w, o, pad, off):
    """Whole numbers: a product with a power of two and every sum are exact in fp32, and so is one rounding to the result's type."""
    g = gen(n + dim)
    tokens = torch.randint(-3, vocab + 3, (n,), generator=g, device="cuda")
    tokens[torch.rand(n, generator=g, device="cuda") < 0.2] = vocab // 2
    held = (tokens >= 0) & (tokens < vocab)
    whole = lambda *s: torch.randint(-8, 9, s, generator=g, device="cuda").float()  # noqa: E731
    table, out = Guarded(vocab, dim, DT[w][0], pad, off, whole(vocab, dim)), Guarded(n, dim, DT[o][0], pad, off)
    LC.lc_embedding_forward(table.matrix(), tokens.data_ptr(), LC.LC_IT_I64, n, out.matrix(), scale=0.5, stream=stream())
    ref = torch.zeros(n, dim, device="cuda")
    ref[held] = table.view.float()[tokens[held]] * 0.5
    assert torch.equal(out.view, ref.to(DT[o][0])) and out.intact()
    dout = Guarded(n, dim, DT[w][0], pad, off, whole(n, dim))
    need = LC.lc_embedding_backward_workspace(n, dim)
    for accumulate in (False, True):
        old = whole(vocab, dim) if accumulate else torch.full((vocab, dim), math.nan, device="cuda")
        dw = Guarded(vocab, dim, DT[o][0], pad, off, old)
        buf, ws, _ = space(need)
        LC.lc_embedding_backward(dout.matrix(), tokens.data_ptr(), LC.LC_IT_I64, n, dw.matrix(), ws, need, scale=0.5,
                                 accumulate=accumulate, stream=stream())
        ref = torch.zeros(vocab, dim, device="cuda").index_add_(0, tokens[held], dout.view.float()[held]) * 0.5 + (old if accumulate else 0)
        assert torch.equal(dw.view, ref.to(DT[o][0]))
        assert dw.intact() and dout.intact() and bool((buf[need:] == 0xA5).all())
