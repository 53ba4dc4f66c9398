"""The weight gradient at sizes that take each of its kernels, with what must not be read made of NaN: the rows
behind the last one, the gaps between rows and what lies before the first.

dY and the kept X are whole numbers (X times a power of two), and no sum of theirs reaches 2^24: every sum is exact in any
order, and the results have to be equal bit for bit."""
import math

import numpy as np
import pytest
import torch

from paper_2609_27193_amd import layercheck as LC
from tests.wgrad_cases import ALIGNED, RAGGED, SMALL

pytestmark = pytest.mark.gpu

BF, F32 = LC.LC_DT_BF16, LC.LC_DT_F32


def among_nan(value, pattern, pad, off):
    """`value` as a view at element `off`, rows `pad` apart, 64 rows of `pattern` behind them: (view, address, stride)."""
    rows, cols = value.shape
    stride = cols + pad
    flat = torch.full((off + (rows + 64) * stride,), pattern, dtype=value.dtype, device="cuda")
    view = flat[off:off + rows * stride].view(rows, stride)[:, :cols]
    view.copy_(value)
    return view, flat.data_ptr() + off * flat.element_size(), stride


def code_of(numbers):
    """Codes of whole numbers from -15 to 15, which the 8-bit form holds exactly."""
    code = np.zeros(16, np.uint8)
    for v in range(1, 16):
        e = int(math.log2(v))
        code[v] = (e + 7) * 8 + (v * 8 // 2 ** e - 8)
    code = torch.from_numpy(code).cuda()[numbers.abs()]
    return torch.where(numbers < 0, code + 128, code).to(torch.uint8)


class Case:
    """dY and X of a size; X is `x` times 2^(scale - 127)."""

    def __init__(self, rows, n, k, pad, off, scale, dtype=torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(rows + n + k)
        self.rows, self.n, self.k, self.power = rows, n, k, 2.0 ** (scale - 127)
        self.d = torch.randint(-3, 4, (rows, n), generator=g, device="cuda")
        self.x = torch.randint(1, 16, (rows, k), generator=g, device="cuda") * (torch.randint(0, 2, (rows, k), generator=g, device="cuda") * 2 - 1)
        self.dy = among_nan(self.d.to(dtype), math.nan, pad, off)
        self.codes = among_nan(code_of(self.x), 127, pad, off)
        self.scales = among_nan(torch.full((rows, -(-k // 32)), scale, dtype=torch.uint8, device="cuda"), 255, pad, off)

    def wgrad(self, **kw):
        need = LC.lc_linear_wgrad_workspace(self.rows, self.n, self.k)
        space = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN, where a part is not written
        dw = torch.full((self.n, self.k), math.nan, device="cuda")
        LC.lc_linear_wgrad(LC.matrix(self.dy[1], self.rows, self.n, BF if self.dy[0].dtype == torch.bfloat16 else F32, self.dy[2]),
                           LC.saved_act(self.codes[1], self.scales[1], self.rows, self.k, self.codes[2], self.scales[2]),
                           LC.matrix(dw.data_ptr(), self.n, self.k, F32), space.data_ptr(), need,
                           stream=torch.cuda.current_stream().cuda_stream, **kw)
        return dw

    def reference(self):
        return (self.dy[0].double().t() @ self.x.double()) * self.power


PLACES = [(0, 0), (0, 1), (3, 1), (24, 8)]


@pytest.mark.parametrize("rows,n,k", [size for size, _ in ALIGNED])
@pytest.mark.parametrize("pad,off", PLACES)
def test_whole_groups(rows, n, k, pad, off):
    c = Case(rows, n, k, pad, off, 130)
    assert torch.equal(c.wgrad().double(), c.reference())


@pytest.mark.parametrize("rows,n,k", [size for size, _ in SMALL])
@pytest.mark.parametrize("pad,off", PLACES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tiles_of_128(rows, n, k, pad, off, dtype):
    c = Case(rows, n, k, pad, off, 120, dtype)
    assert torch.equal(c.wgrad().double(), c.reference())


@pytest.mark.parametrize("rows,n,k", [size for size, _ in RAGGED])
@pytest.mark.parametrize("pad,off", PLACES)
def test_every_token_is_counted_once(rows, n, k, pad, off):
    """X near the smallest of the 8-bit form's powers, of which a token taken again with a scale of zero shows."""
    c = Case(rows, n, k, pad, off, 8)
    assert torch.equal(c.wgrad().double(), c.reference())


@pytest.mark.parametrize("rows,n,k", [size for size, _ in RAGGED])
@pytest.mark.parametrize("pad", [0, 3])
def test_an_infinity_of_the_last_token_stays_one(rows, n, k, pad):
    """X holds no zero, so an infinity of dY times it is one, in its row of dW and in no other."""
    c = Case(rows, n, k, pad, 0, 127)
    for col, v in ((0, math.inf), (5, -math.inf), (7, math.inf), (n - 1, -math.inf)):
        c.dy[0][-1, col] = v
    got, want = c.wgrad().double(), c.reference()
    assert bool(torch.isinf(want[0]).all()) and int(torch.isinf(want).any(1).sum()) == 4
    assert torch.equal(got, want)
