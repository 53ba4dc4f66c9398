"""The weight gradient at sizes that take each of its kernels, with what must not be read made of NaN: the rows
behind the last one, the gaps between rows and what lies before the first.

dY and the kept X are whole numbers (X times a power of two), and no sum of theirs reaches 2^24: every sum is exact in any
order, and the results have to be equal bit for bit."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2609_27193_amd import layercheck as LC
from paper_2609_27193_amd.build_lib import GRID_CAPPED_LIB
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
@pytest.mark.parametrize("pad,off", PLACES[1:3])
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


@pytest.mark.parametrize("rows,n,k", [size for size, _ in RAGGED + ALIGNED + SMALL])
@pytest.mark.parametrize("out,param", [("bf16", "f32"), ("f32", "bf16")])
def test_scale_shift_bias_and_what_is_there(rows, n, k, out, param):
    """Scales of 1/2, 1 and 2 and whole shifts: what is added to dW and to the bias's gradient is exact in fp32 as well, and
    is rounded to their type once."""
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    c = Case(rows, n, k, 0, 1, 127)
    g = torch.Generator(device="cuda").manual_seed(k)
    scale = torch.exp2(torch.randint(-1, 2, (k,), generator=g, device="cuda").float()).to(types[param])
    shift = torch.randint(-2, 3, (k,), generator=g, device="cuda").to(types[param])
    sums = c.d.double().sum(0)
    want = c.reference() * scale.double() + sums[:, None] * shift.double()
    assert bool((want.abs() < 2 ** 22).all())
    code = {torch.bfloat16: BF, torch.float32: F32}
    need = LC.lc_linear_wgrad_workspace(rows, n, k)
    space = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    for accumulate in (False, True):
        for bias in (False, True):
            old, old_b = (torch.randint(-9, 10, s, generator=g, device="cuda").to(types[out]) for s in ((n, k), (n,)))
            dw, db = (old.clone(), old_b.clone()) if accumulate else (torch.full_like(old, math.nan), torch.full_like(old_b, math.nan))
            LC.lc_linear_wgrad(LC.matrix(c.dy[1], rows, n, BF, c.dy[2]),
                               LC.saved_act(c.codes[1], c.scales[1], rows, k, c.codes[2], c.scales[2]),
                               LC.matrix(dw.data_ptr(), n, k, code[dw.dtype]), space.data_ptr(), need, col_scale=scale.data_ptr(),
                               col_shift=shift.data_ptr(), param_dtype=code[scale.dtype], dbias=db.data_ptr() if bias else 0,
                               accumulate=accumulate, stream=torch.cuda.current_stream().cuda_stream)
            base, base_b = (old.double(), old_b.double()) if accumulate else (0, 0)
            assert torch.equal(dw, (want + base).float().to(types[out]))
            if bias:
                assert torch.equal(db, (sums + base_b).float().to(types[out]))


@pytest.mark.parametrize("rows,n,k", [(513, 2565, 4095), (4110, 2565, 1790), (513, 2568, 4096), (33, 257, 130), (95, 300, 15)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scales_at_both_ends(rows, n, k, dtype):
    """A scale byte of 0 is 2^-127, of 255 NaN, in its 32 columns of X and in no others; a NaN code in its column."""
    c = Case(rows, n, k, 0, 1, 0, dtype)
    c.dy[0].copy_(c.d.clamp(min=1).double() * 2.0 ** 30)  # no zero times NaN, and sums of normal fp32 size
    want = (c.dy[0].double().t() @ c.x.double()) * 2.0 ** -127
    last = -(-k // 32) - 1
    c.scales[0][rows // 2, last] = 255
    c.codes[0][rows - 1, 3] = 255
    want[:, last * 32:] = math.nan
    want[:, 3] = math.nan
    got = c.wgrad().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(want))


@pytest.mark.parametrize("n,k", [(4096, 4096), (2565, 4095), (9, 17)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_tokens(n, k, dtype):
    """Zeros, or what is there; dY and X have no rows and need no address."""
    need = LC.lc_linear_wgrad_workspace(0, n, k)
    space = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    scale, shift = torch.full((k,), 2.0, device="cuda"), torch.full((k,), 3.0, device="cuda")
    for accumulate, before, after in ((False, math.nan, 0.0), (True, 5.0, 5.0)):
        dw, db = torch.full((n, k), before, device="cuda"), torch.full((n,), before, device="cuda")
        LC.lc_linear_wgrad(LC.matrix(0, 0, n, dtype), LC.saved_act(0, 0, 0, k), LC.matrix(dw.data_ptr(), n, k, F32),
                           space.data_ptr(), need, col_scale=scale.data_ptr(), col_shift=shift.data_ptr(), dbias=db.data_ptr(),
                           accumulate=accumulate, stream=torch.cuda.current_stream().cuda_stream)
        assert bool((dw == after).all()) and bool((db == after).all())


def test_grids_capped_at_forty_blocks():
    """Blocks that take several tiles, and several parts, after each other."""
    if not os.path.exists(GRID_CAPPED_LIB):
        pytest.skip("the grid-capped library is built by __graft_entry__.build()")
    if os.environ.get("LAYERCHECK_LIB"):
        pytest.skip("runs in the parent only")
    pick = "(token or groups or there) and (513 or 4097 or 4110 or 16385 or 8200 or 4099)"
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "-m", "gpu", "-k", pick,
                        os.path.abspath(__file__)], env=dict(os.environ, LAYERCHECK_LIB=GRID_CAPPED_LIB),
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True,
                       timeout=600)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
