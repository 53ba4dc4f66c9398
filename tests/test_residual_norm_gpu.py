"""The norm with the residual's addition against plain implementations in 64 bits, and against the norm alone bit for bit.

As in the norm's tests, U32 = 2^-24 stands for a rounding of an fp32 operation and an addend of a row's sum passes norm_depth
additions; the sum x + residual is one more rounding of each element (SUM more in each bound: the element's own and what it
does to mean and rstd)."""
import math

import pytest
import torch

from paper_2609_27193_amd import layercheck as LC
from tests.test_operators_gpu import (DT, U32, Guarded, Kept, close, gen, keep, kept_normal, norm_depth, norm_reference,
                                      norm_sums_depth, space, stream)

pytestmark = pytest.mark.gpu

SUM = 4
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]  # of x and y, of the residual and h
SIZES = [(0, 8), (1, 1), (3, 2), (5, 7), (4, 8), (9, 31), (2, 96), (7, 511), (6, 512), (5, 513), (3, 1024), (9, 1027), (3, 2048),
         (4, 2050), (2, 4096), (3, 5120), (2, 6145), (3, 8192), (2, 8200), (2, 16384), (2, 16391), (1, 40003), (700, 64),
         (1200, 160), (9000, 520), (900, 16384)]


def params(rms, w, b, code, eps=1e-5):
    return LC.norm_params(LC.LC_NORM_RMS if rms else LC.LC_NORM_LAYER, w.data_ptr(), 0 if rms else b.data_ptr(), code, eps)


def near_8_bits(k, ref, tol):
    """Values kept in 8 bits lie next to ref: half a step of its 4 bits, or of the block's smallest step, and ref's own error."""
    rows, dim = ref.shape
    step = torch.ldexp(torch.ones_like(ref), (k.scales.view.long() - 127 - 10).repeat_interleave(32, 1)[:, :dim])
    close(k.values(), ref, torch.maximum(ref.abs() / 16, step) * (1 + 1e-6) + 2 * tol)


@pytest.mark.parametrize("rows,dim", SIZES)
@pytest.mark.parametrize("dtype,res", TYPES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_forward(rows, dim, dtype, res, kind):
    rms = kind == "rms"
    dt, _, u_out = DT[dtype]
    rt = DT[res][0]
    g = gen(rows + 31 * dim)
    pad, off = (5, 1) if dim % 2 else (8, 3) if rows == 3 else (0, 0)
    x = Guarded(rows, dim, dt, pad, off, torch.randn(rows, dim, generator=g, device="cuda"))
    r = Guarded(rows, dim, rt, pad, off, torch.randn(rows, dim, generator=g, device="cuda") * 3 + 0.5)
    w = (1 + 0.3 * torch.randn(dim, generator=g, device="cuda")).to(dt)
    b = torch.zeros(dim, device="cuda") if rms else (0.3 * torch.randn(dim, generator=g, device="cuda")).to(dt)
    prm = params(rms, w, b, DT[dtype][1])

    def call(h=True, y=True, saved=True, y_saved=True, stats=True):
        out = dict(h=Guarded(rows, dim, rt, pad, off) if h else None, y=Guarded(rows, dim, dt, pad, off) if y else None,
                   mean=torch.empty(rows + 1, device="cuda"), rstd=torch.empty(rows + 1, device="cuda"),
                   saved=Kept(rows, dim, pad=pad, off=off) if saved else None, y_saved=Kept(rows, dim, pad=pad, off=off) if y_saved else None)
        LC.lc_residual_norm_forward(prm, x.matrix(), r.matrix(), out["h"].matrix() if h else None, out["y"].matrix() if y else None,
                                    out["mean"].data_ptr() if stats and not rms else 0, out["rstd"].data_ptr() if stats else 0,
                                    out["saved"].act if saved else None, out["y_saved"].act if y_saved else None, stream())
        for name in ("h", "y", "saved", "y_saved"):
            assert out[name] is None or out[name].intact()
        return out

    out = call()
    assert x.intact() and r.intact()
    assert torch.equal(out["h"].view, (x.view.float() + r.view.float()).to(rt))  # one addition, one rounding
    if rows:
        h = x.view.double() + r.view.double()
        rm, rr, rn, ry = norm_reference(h, w, b, rms, 1e-5)
        depth = norm_depth(dim) + SUM
        size = h.abs().mean(1, keepdim=True)
        shift = depth * U32 * size * (0 if rms else 1)
        if not rms:
            close(out["mean"][:rows], rm[:, 0], depth * U32 * size[:, 0])
        # a sum's rounding counts against the spread (dim 1: none is left)
        spread = U32 * h.abs().amax(1, keepdim=True) * (0 if rms else 1)
        close(out["rstd"][:rows], rr[:, 0], (depth * U32 * rr + (shift + spread) ** 2 * rr ** 3 + spread * rr ** 2)[:, 0])
        n_tol = depth * U32 * rn.abs() + (shift + U32 * h.abs()) * rr + 2 * U32 * rm.abs() * rr + rn.abs() * spread * rr
        y_tol = n_tol * w.double().abs() + 4 * U32 * (ry.abs() + b.double().abs())
        close(out["y"].view, ry, 2 * u_out * ry.abs() + y_tol)
        near_8_bits(out["saved"], rn, n_tol)
        near_8_bits(out["y_saved"], ry, y_tol)
        if dtype == "f32":  # y as it is, in 8 bits
            codes, scales = keep(out["y"].view.cpu()) if rows * dim < 20000 else (None, None)
            k = Kept(rows, dim)
            LC.lc_act_save(out["y"].matrix(), k.act, stream())
            assert torch.equal(k.codes.view, out["y_saved"].codes.view) and torch.equal(k.scales.view, out["y_saved"].scales.view)
            assert codes is None or (torch.equal(k.codes.view.cpu(), codes) and torch.equal(k.scales.view.cpu(), scales))
    # parts of it: the same bits
    for part in (dict(h=False, saved=False, stats=False), dict(y=False, saved=False), dict(h=False, y_saved=False)):
        again = call(**part)
        for name in ("h", "y"):
            assert again[name] is None or torch.equal(again[name].view, out[name].view)
        for name in ("saved", "y_saved"):
            assert again[name] is None or (torch.equal(again[name].codes.view, out[name].codes.view)
                                           and torch.equal(again[name].scales.view, out[name].scales.view))


@pytest.mark.parametrize("dim", [5, 64, 1100, 4096, 6000, 16390])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_a_residual_alone_is_the_norm(dim, kind):
    """x of zeros: the bits of lc_norm_forward."""
    rows, rms = 11, kind == "rms"
    g = gen(dim)
    r = Guarded(rows, dim, torch.float32, 3, 1, torch.randn(rows, dim, generator=g, device="cuda"))
    x = Guarded(rows, dim, torch.float32, value=torch.zeros(rows, dim))
    w, b = (torch.randn(dim, generator=g, device="cuda") for _ in "wb")
    prm = params(rms, w, b, LC.LC_DT_F32)
    y, y2, h = (Guarded(rows, dim, torch.float32) for _ in range(3))
    k, k2 = Kept(rows, dim), Kept(rows, dim)
    st = torch.empty(4, rows, device="cuda")
    LC.lc_norm_forward(prm, r.matrix(), y.matrix(), 0 if rms else st[0].data_ptr(), st[1].data_ptr(), k.act, stream())
    LC.lc_residual_norm_forward(prm, x.matrix(), r.matrix(), h.matrix(), y2.matrix(), 0 if rms else st[2].data_ptr(),
                                st[3].data_ptr(), k2.act, stream=stream())
    assert torch.equal(y.view, y2.view) and torch.equal(h.view, r.view) and torch.equal(st[1], st[3])
    assert torch.equal(k.codes.view, k2.codes.view) and torch.equal(k.scales.view, k2.scales.view)
    assert rms or torch.equal(st[0], st[2])


@pytest.mark.parametrize("dtype,res", TYPES)
@pytest.mark.parametrize("dim", [40, 1500, 9000, 17000])
def test_edges(dtype, res, dim):
    """A row of zeros, rows that hold an infinity or a NaN, in either addend, and infinities that meet: the rows beside are as
    ever, and the 8-bit form of a row that is all NaN is NaN."""
    g = gen(dim)
    dt, rt = DT[dtype][0], DT[res][0]
    x, r = torch.randn(7, dim, generator=g, device="cuda"), torch.randn(7, dim, generator=g, device="cuda")
    x[1], r[1] = 0, 0
    x[2, 3], r[3, dim - 1] = math.nan, math.inf
    x[4, 5], r[4, 5] = math.inf, -math.inf
    X, R = Guarded(7, dim, dt, value=x), Guarded(7, dim, rt, value=r)
    w = torch.ones(dim, dtype=dt, device="cuda")
    for rms in (True, False):
        b = torch.zeros(dim, dtype=dt, device="cuda")
        prm = params(rms, w, b, DT[dtype][1])
        y, h, k, y8 = Guarded(7, dim, dt), Guarded(7, dim, rt), Kept(7, dim), Kept(7, dim)
        LC.lc_residual_norm_forward(prm, X.matrix(), R.matrix(), h.matrix(), y.matrix(), saved=k.act, y_saved=y8.act, stream=stream())
        assert torch.equal(torch.isnan(h.view), torch.isnan(X.view.float() + R.view.float()))
        nan_rows = torch.isnan(y.view).all(1).tolist()
        assert nan_rows[2] and nan_rows[4] and not any(nan_rows[i] for i in (0, 1, 5, 6))
        assert torch.isnan(y.view[3, dim - 1]).item()  # inf / inf
        assert not bool(y.view[1].any()) and not bool(k.values()[1].any()) and not bool(y8.values()[1].any())
        for v in (k.values(), y8.values()):
            assert bool(torch.isnan(v[[2, 4]]).all()) and bool(torch.isfinite(v[[0, 1, 5, 6]]).all())
        part = [0, 5, 6]
        X2, R2 = Guarded(3, dim, dt, value=X.view[part]), Guarded(3, dim, rt, value=R.view[part])
        y2, k2 = Guarded(3, dim, dt), Kept(3, dim)
        LC.lc_residual_norm_forward(prm, X2.matrix(), R2.matrix(), None, y2.matrix(), saved=k2.act, stream=stream())
        assert torch.equal(y2.view, y.view[part]) and torch.equal(k2.values(), k.values()[part])


@pytest.mark.parametrize("rows,dim", SIZES)
@pytest.mark.parametrize("dtype,res", TYPES)
@pytest.mark.parametrize("kind,source", [("rms", "h"), ("rms", "kept"), ("layer", "h"), ("layer", "kept")])
def test_gradient(rows, dim, dtype, res, kind, source):
    rms = kind == "rms"
    dt, _, u_out = DT[dtype]
    rt, _, u_res = DT[res]
    gt, gcode, u_grad = DT["bf16" if dim % 3 else "f32"]
    g = gen(rows + 17 * dim)
    pad, off = (5, 1) if dim % 2 else (8, 3) if rows == 3 else (0, 0)
    dy = Guarded(rows, dim, dt, pad, off, torch.randn(rows, dim, generator=g, device="cuda"))
    dh = Guarded(rows, dim, rt, pad, off, torch.randn(rows, dim, generator=g, device="cuda"))
    w = (1 + 0.3 * torch.randn(dim, generator=g, device="cuda")).to(dt)
    rstd = torch.rand(rows + 1, generator=g, device="cuda") + 0.5
    mean = torch.randn(rows + 1, generator=g, device="cuda")
    rs = rstd[:rows, None].double()
    h = k = None
    if source == "h":
        h = Guarded(rows, dim, rt, pad, off, torch.randn(rows, dim, generator=g, device="cuda"))
        m64 = mean[:rows, None].double() * (0 if rms else 1)
        n = (h.view.double() - m64) * rs
        n_tol = 3 * U32 * (n.abs() + m64.abs() * rs)
    else:
        k = kept_normal(rows, dim, dim, pad, off)
        n = k.values()
        n_tol = torch.zeros_like(n)
    prm = LC.norm_params(LC.LC_NORM_RMS if rms else LC.LC_NORM_LAYER, w.data_ptr(), 0, DT[dtype][1], 1e-5)
    need = LC.lc_norm_backward_workspace(rows, dim)
    d64 = dy.view.double()
    gw = d64 * w.double()
    c1 = gw.mean(1, keepdim=True) * (0 if rms else 1) if rows else torch.zeros(0, 1, dtype=torch.float64, device="cuda")
    c2 = (gw * n).mean(1, keepdim=True)
    part = rs * (gw - c1 - n * c2)
    want_dx = dh.view.double() + part
    depth = norm_depth(dim)
    c1_tol = depth * U32 * gw.abs().mean(1, keepdim=True) * (0 if rms else 1)
    c2_tol = depth * U32 * (gw * n).abs().mean(1, keepdim=True) + (gw.abs() * n_tol).mean(1, keepdim=True)
    dx_tol = rs * (4 * U32 * (gw.abs() + c1.abs() + (n * c2).abs()) + c1_tol + n.abs() * c2_tol + n_tol * c2.abs()) + U32 * want_dx.abs()
    rw, rb = (d64 * n).sum(0), d64.sum(0)
    args = dict(h=h.matrix() if h else None, mean=mean.data_ptr() if h and not rms else 0, saved=k.act if k else None, stream=stream())
    for accumulate in (False, True):
        dx, dres = Guarded(rows, dim, dt, pad, off), Guarded(rows, dim, rt, pad, off)
        old_w, old_b = (torch.randn(1, dim, generator=g, device="cuda") for _ in "wb")
        dw = Guarded(1, dim, gt, 0, off, old_w if accumulate else torch.full_like(old_w, math.nan))
        db = Guarded(1, dim, gt, 0, off, old_b if accumulate else torch.full_like(old_b, math.nan))
        buf, ws, _ = space(need)
        LC.lc_residual_norm_backward(prm, dy.matrix(), dh.matrix(), rstd.data_ptr(), dx.matrix(), dres.matrix(), dw.addr,
                                     0 if rms else db.addr, gcode, ws, need, accumulate=accumulate, **args)
        assert bool((buf[need:] == 0xA5).all())
        if rows:
            close(dx.view, want_dx, 2 * u_out * want_dx.abs() + dx_tol)
            close(dres.view, want_dx, 2 * u_res * want_dx.abs() + dx_tol)
            assert torch.equal(dres.view.to(dt), dx.view)  # one gradient, in two types
        sd = norm_sums_depth(rows)
        for got, want, size, old in ((dw, rw, (d64 * n).abs().sum(0) + (d64.abs() * n_tol).sum(0) / (sd * U32), old_w),
                                     (db, rb, d64.abs().sum(0), old_b)):
            if got is db and rms:
                continue
            base = old.to(gt).double()[0] if accumulate else torch.zeros_like(want)
            close(got.view[0], want + base, 2 * u_grad * (want + base).abs() + sd * U32 * size * (1 + u_grad) + 2 * U32 * base.abs())
        assert all(t.intact() for t in (dx, dres, dw, dy, dh)) and (rms or db.intact())
    # parts of it: the same bits
    dx2, dres2 = Guarded(rows, dim, dt, pad, off), Guarded(rows, dim, rt, pad, off)
    LC.lc_residual_norm_backward(prm, dy.matrix(), dh.matrix(), rstd.data_ptr(), dx2.matrix(), None, 0, 0, gcode, 0, 0, **args)
    LC.lc_residual_norm_backward(prm, dy.matrix(), dh.matrix(), rstd.data_ptr(), None, dres2.matrix(), 0, 0, gcode, 0, 0, **args)
    assert torch.equal(dx2.view, dx.view) and torch.equal(dres2.view, dres.view)
    dw2 = Guarded(1, dim, gt, 0, off, old_w)
    LC.lc_residual_norm_backward(prm, dy.matrix(), dh.matrix(), rstd.data_ptr(), None, None, dw2.addr, 0, gcode, ws, need,
                                 accumulate=True, **args)
    assert torch.equal(dw2.view, dw.view)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradient_against_differences(kind):
    """loss = sum dy * y + sum dh * h, whose gradient the call gives; central differences of the 64-bit formula are off by their
    step's square (1e-6 of third derivatives of order one, times the 200 columns' part) and the forward's statistics by fp32."""
    rms, rows, dim, eps = kind == "rms", 6, 200, 1e-3
    g = gen(11)
    x, r, dy, dh = (torch.randn(rows, dim, generator=g, device="cuda") for _ in range(4))
    w = 1 + 0.3 * torch.randn(dim, generator=g, device="cuda")
    b = torch.randn(dim, generator=g, device="cuda")
    prm = params(rms, w, b, LC.LC_DT_F32, eps)
    m = lambda t: LC.matrix(t.data_ptr(), rows, dim, LC.LC_DT_F32)  # noqa: E731
    y, h, dx = (torch.empty_like(x) for _ in range(3))
    st = torch.empty(2, rows, device="cuda")
    dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    LC.lc_residual_norm_forward(prm, m(x), m(r), m(h), m(y), 0 if rms else st[0].data_ptr(), st[1].data_ptr(), stream=stream())
    need = LC.lc_norm_backward_workspace(rows, dim)
    buf, ws, _ = space(need)
    LC.lc_residual_norm_backward(prm, m(dy), m(dh), st[1].data_ptr(), m(dx), None, dw.data_ptr(), 0 if rms else db.data_ptr(),
                                 LC.LC_DT_F32, ws, need, h=m(h), mean=0 if rms else st[0].data_ptr(), stream=stream())

    def loss(x, r, w, b):
        s = x.double() + r.double()
        y = norm_reference(s, w, torch.zeros_like(b) if rms else b, rms, eps)[3]
        return ((dy.double() * y).sum() + (dh.double() * s).sum()).item()

    step = 1e-3
    for name, at, grad in [("x", 0, dx), ("r", 1, dx), ("w", 2, dw)] + ([] if rms else [("b", 3, db)]):
        for i in range(0, grad.numel(), 97):
            args = [x.double(), r.double(), w.double(), b.double()]
            args[at] = args[at].clone()
            args[at].view(-1)[i] += step
            up = loss(*args)
            args[at].view(-1)[i] -= 2 * step
            diff = (up - loss(*args)) / (2 * step)
            assert abs(diff - grad.view(-1)[i].item()) <= 2e-5 * (1 + abs(diff)), (name, i)


def block(rows, dim, seed):
    """A pre-norm block's calls around a linear layer as a training step makes them: (enqueue, results, what they read)."""
    g = gen(seed)
    bf = torch.bfloat16
    E = lambda *s, dtype=bf: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    M = lambda t: LC.matrix(t.data_ptr(), t.shape[0], t.shape[1], LC.LC_DT_BF16 if t.dtype == bf else LC.LC_DT_F32)  # noqa: E731
    x, dy = (torch.randn(rows, dim, generator=g, device="cuda").to(bf) for _ in "xd")
    r, dh = (torch.randn(rows, dim, generator=g, device="cuda") for _ in "rd")
    dz = torch.randn(rows, 96, generator=g, device="cuda").to(bf)
    w = torch.rand(dim, generator=g, device="cuda").to(bf)
    h, dres, y, dx, dlin = E(rows, dim, dtype=torch.float32), E(rows, dim, dtype=torch.float32), E(rows, dim), E(rows, dim), E(96, dim)
    rstd, dw = E(rows, dtype=torch.float32), E(dim, dtype=torch.float32)
    codes, scales = E(rows, dim, dtype=torch.uint8), E(rows, -(-dim // 32), dtype=torch.uint8)
    y8 = LC.saved_act(codes.data_ptr(), scales.data_ptr(), rows, dim)
    need = max(LC.lc_norm_backward_workspace(rows, dim), LC.lc_linear_wgrad_workspace(rows, 96, dim))
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    prm = LC.norm_params(LC.LC_NORM_RMS, w.data_ptr(), 0, LC.LC_DT_BF16, 1e-5)

    def enqueue():
        s = stream()
        LC.lc_residual_norm_forward(prm, M(x), M(r), M(h), M(y), rstd=rstd.data_ptr(), y_saved=y8, stream=s)
        LC.lc_linear_wgrad(M(dz), y8, M(dlin), ws.data_ptr(), need, stream=s)
        LC.lc_residual_norm_backward(prm, M(dy), M(dh), rstd.data_ptr(), M(dx), M(dres), dw.data_ptr(), 0, LC.LC_DT_F32,
                                     ws.data_ptr(), need, h=M(h), stream=s)

    return enqueue, [h, y, rstd, codes, scales, dlin, dx, dres, dw], (x, dy, r, dh, dz, w, ws)


def test_the_8_bit_rows_feed_the_weight_gradient():
    """dW from y_saved is dz^T y to within 4 bits of each y: 2^-4 of the products' magnitudes, and dW's own rounding."""
    enqueue, res, (x, dy, r, dh, dz, w, _) = block(300, 136, 4)
    enqueue()
    h = x.double() + r.double()
    y = h / torch.sqrt(h.square().mean(1, keepdim=True) + 1e-5) * w.double()
    want, size = dz.double().t() @ y, dz.double().abs().t() @ y.abs()
    close(res[5], want, 2.0 ** -4 * size + 2.0 ** -7 * want.abs() + 2.0 ** -17 * dz.double().abs().sum(0)[:, None] * y.abs().max())


@pytest.mark.parametrize("rows", [3, 5000])
def test_calls_in_a_graph(rows):
    enqueue, results, keepalive = block(rows, 264, 1)
    enqueue()
    torch.cuda.synchronize()
    want = [r.clone() for r in results]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        enqueue()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            enqueue()
    for i in range(4):
        for r in results:
            r.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want)), i


def test_offsets_beyond_32_bits():
    """Rows of more than 2^32 bytes: the last ones are those of the same rows alone, bit for bit."""
    rows, dim = (1 << 18) + 40, 8192
    g = gen(5)
    x = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    x[-40:] = torch.randn(40, dim, generator=g, device="cuda")
    r, h, y = x.clone(), torch.empty_like(x), torch.empty_like(x)
    w = torch.ones(dim, dtype=torch.bfloat16, device="cuda")
    rstd = torch.empty(rows, device="cuda")
    prm = LC.norm_params(LC.LC_NORM_RMS, w.data_ptr(), 0, LC.LC_DT_BF16, 1e-5)
    M = lambda t: LC.matrix(t.data_ptr(), t.shape[0], dim, LC.LC_DT_BF16)  # noqa: E731
    LC.lc_residual_norm_forward(prm, M(x), M(r), M(h), M(y), rstd=rstd.data_ptr(), stream=stream())
    few = [t[-40:].clone() for t in (x, r)]
    h2, y2 = torch.empty_like(few[0]), torch.empty_like(few[0])
    LC.lc_residual_norm_forward(prm, M(few[0]), M(few[1]), M(h2), M(y2), stream=stream())
    assert torch.equal(h[-40:], h2) and torch.equal(y[-40:], y2) and bool(y2.any())
    dx = torch.empty_like(x)
    LC.lc_residual_norm_backward(prm, M(y), M(x), rstd.data_ptr(), M(dx), None, 0, 0, LC.LC_DT_F32, 0, 0, h=M(h), stream=stream())
    dx2, rs = torch.empty_like(h2), rstd[-40:].clone()
    LC.lc_residual_norm_backward(prm, M(y2), M(few[0]), rs.data_ptr(), M(dx2), None, 0, 0, LC.LC_DT_F32, 0, 0, h=M(h2), stream=stream())
    assert torch.equal(dx[-40:], dx2)
