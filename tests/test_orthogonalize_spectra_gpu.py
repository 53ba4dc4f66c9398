"""What the orthogonalised update is off by on matrices whose singular values are far apart, as an optimizer's are: few large ones
and a long tail.  The steps raise the small ones by up to a^5, some 480, and with them whatever noise lies in their directions.

The bound is the error of the held precision itself, on the same matrix: the steps in 64 bits with X rounded to 22 bits, A and
B = b A + c A A to 11 (a result in fp32 or of a shorter side below 384: to 22) and the products taken from X's first 11.  The
kernel's roundings are others of the same sizes, so its error is held to one and a half times that (a sum of thousands of
roundings differs from another such sum by a few percent), plus twice the error of the formula in fp32 throughout, for sums in
fp32 (of three products, one addend after the other), plus the rounding of a bf16 result (that of the exact result, and a tenth for
its being another value that is rounded).  The identity's elements are one number, whose rounding to bf16 is no sum of many but one
rounding, up to 2^-8: of 512 x 1024 the exact 0.808607 goes to 0.808594, off by 1.6e-5, and the steps' 0.806162, off by 3.0e-3 with 11
bits, to 0.804688, off by 4.8e-3.  (In fp32 every rounding of its steps is such a single one, and no sum of others of that size says how
large it may be.)"""
import pytest
import torch

from tests.test_operators_gpu import Guarded, gen
from tests.test_orthogonalize_bounds import SHARP
from tests.test_orthogonalize_gpu import CUBIC, STEEP, call, whole

pytestmark = pytest.mark.gpu

ONE_PLANE = 384  # a bf16 result's A and B are of 11 bits from this shorter side on
KINDS = ["normal", "alike", "identity", "1/i", "1/i^2", "exp(-i/40)", "eight and a tail", "rank 1", "rank 4", "rank 16", "rank 64"]


def matrix(rows, cols, kind, seed=0):
    """rows x cols in fp32 with such singular values."""
    g = gen(1000 + rows + cols + seed)
    m, n = min(rows, cols), max(rows, cols)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
    if kind == "normal":
        x = randn(m, n)
    elif kind == "alike":
        x = torch.linalg.qr(randn(n, m))[0].t()
    elif kind == "identity":
        x = torch.eye(m, n, device="cuda", dtype=torch.float64)
    elif kind.startswith("rank"):
        r = min(int(kind[5:]), m)
        x = randn(m, r) @ randn(r, n)
    else:
        i = torch.arange(1, m + 1, device="cuda", dtype=torch.float64)
        values = {"1/i": 1 / i, "1/i^2": 1 / i ** 2, "exp(-i/40)": torch.exp(-i / 40),
                  "eight and a tail": torch.where(i <= 8, torch.ones_like(i), torch.full_like(i, 1e-4))}[kind]
        x = (torch.linalg.qr(randn(m, m))[0] * values) @ torch.linalg.qr(randn(n, m))[0].t().contiguous()
    return (x.t() if rows > cols else x).float().contiguous()


def held(x, planes):
    """x in 11 bits or 22: an fp16 number near 2^15 and the rest, 2^11 times as large, in another."""
    power = 2.0 ** (14 - torch.floor(torch.log2(x.abs().max()))) if bool(x.any()) else 1.0
    hi = (x * power).half().double()
    return (hi if planes == 1 else hi + ((x * power - hi) * 2048).half().double() / 2048) / power


def steps(u, coefs, rounded=lambda x, planes: x, planes=2):
    x = u / torch.linalg.vector_norm(u.double()).to(u.dtype)
    x = rounded((x.t() if x.shape[0] > x.shape[1] else x).contiguous(), 2)
    for a, b, c in coefs:
        of = rounded(x, planes)
        gram = rounded(of @ of.t().contiguous(), planes)
        x = rounded(a * x + rounded(b * gram + c * (gram @ gram), planes) @ of, 2)
    return x.t() if u.shape[0] > u.shape[1] else x


def distance(x, want):
    return (torch.linalg.matrix_norm(x.double() - want) / torch.linalg.matrix_norm(want)).item()


def check(rows, cols, kind, out, coefs):
    u = matrix(rows, cols, kind)
    got = call([Guarded(rows, cols, torch.float32, value=u)], out, len(coefs), coefs)[0].view
    want = steps(u.double(), coefs)
    planes = 1 if out == "bf16" and min(rows, cols) >= ONE_PLANE else 2
    bound = 1.5 * distance(steps(u.double(), coefs, held, planes), want) + 2 * distance(steps(u, coefs), want)
    if out == "bf16":
        bound += 2.0 ** -8 if kind == "identity" else 1.1 * distance(want.bfloat16(), want)
    off = distance(got, want)
    print(f"{rows} x {cols} {kind} {out}: {off:.2e}, bound {bound:.2e}")
    assert off <= bound


SIDES = [(16, 16), (40, 300), (383, 512), (384, 384), (512, 1024), (1500, 400), (1100, 1090)]


@pytest.mark.parametrize("rows,cols", SIDES)
@pytest.mark.parametrize("kind,out", [(k, o) for o in ("bf16", "f32") for k in KINDS if (k, o) != ("identity", "f32")])
@pytest.mark.parametrize("coefs", [[STEEP] * 5, [CUBIC] * 5, [(2.0, -1.5, 0.5)] * 8], ids=["steep", "cubic", "quintic"])
def test_few_large_singular_values(rows, cols, kind, out, coefs):
    check(rows, cols, kind, out, coefs)


@pytest.mark.parametrize("rows,cols", [(64, 64), (70, 300), (500, 400)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("tiny", [1e-18, -1e-18, 1e-12])
def test_a_tiny_coefficient(rows, cols, out, tiny):
    """s = 1.698 s, then 1.5 s - 0.5 s^3 + tiny s^5, which has its largest value of 1 inside and ends near its zero, then s: what a step
    holds must not overflow."""
    coefs = [(1.698, 0.0, 0.0), (1.5, -0.5, tiny), (1.0, 0.0, 0.0)]
    check(rows, cols, "normal", out, coefs)


@pytest.mark.parametrize("rows,cols", [(90, 70), (384, 512)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_steps_that_need_their_range(rows, cols, kind, out):
    """Polynomials that turn upwards right behind the range that the step before leaves."""
    if (kind, out) != ("identity", "f32"):
        check(rows, cols, kind, out, SHARP)


@pytest.mark.parametrize("rows,cols,n,dtype", [(2050, 1900, 17, "bf16"), (1000, 60000, 9, "f32"), (4000, 3970, 5, "bf16")])
def test_matrices_in_turns(rows, cols, n, dtype):
    """More matrices than are worked on at once, in turns of 9 and 8, of 5 and 4, of 3 and 2: whole numbers come out exactly."""
    grads = [whole(rows, cols, 6, s, dtype) for s in range(n)]
    outs = call(grads, dtype, 1, (1.0, 1.0, 0.0))
    for g, o in zip(grads, outs):
        x = g.view.double()
        x = (x.t() if rows > cols else x).contiguous()
        gram = x @ x.t().contiguous()
        assert gram.abs().max() <= 2048  # eleven bits
        want = (x + gram @ x / 4.0 ** 6) / 2.0 ** 6
        want = want.t() if rows > cols else want
        assert torch.equal(o.view, want.float().to(o.view.dtype))


def test_a_momentum_without_momenta_has_no_effect():
    grad = Guarded(60, 90, torch.float32, value=matrix(60, 90, "normal"))
    plain = call([grad], "f32", momentum=0.0)[0].view
    for nesterov in (False, True):
        assert torch.equal(call([grad], "f32", momentum=0.95, nesterov=nesterov)[0].view, plain)
