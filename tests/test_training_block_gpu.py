"""The operators of a pre-norm block and of its optimizer together, as a training program calls them: the residual norm in 8 bits,
the weight gradient from those, the norm's gradient, momentum and Newton-Schulz steps of the matrices' gradients with the
momentum in the layout's first moments, the mixed step that takes the results, the decision, the pack and the restore."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2609_27193_amd import layercheck as LC
from paper_2609_27193_amd.build_lib import GRID_CAPPED_LIB
from tests.test_operators_gpu import stream

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
ROWS, DIM, BLOCKS = 200, 136, 3


def M(t):
    return LC.matrix(t.data_ptr(), t.shape[0], t.shape[1], LC.LC_DT_BF16 if t.dtype == BF else LC.LC_DT_F32, t.stride(0))


class Program:
    """Blocks of h_i = h_{i-1} + x_i, y_i = rms(h_i) w_i, x_{i+1} = y_i W_i^T; the loss is half the mean square of the last h's
    distance from a target.  Weights bf16 with fp32 master copies, the residual stream fp32."""

    def __init__(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        E = lambda *s, dtype=F32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
        self.W = [(rnd(DIM, DIM) * 0.1).to(BF) for _ in range(BLOCKS)]
        self.w = [(1 + 0.1 * rnd(DIM)).to(BF) for _ in range(BLOCKS)]
        self.params = [t for pair in zip(self.W, self.w) for t in pair]
        self.master = [t.float().clone() for t in self.params]
        self.m, self.v = ([E(*t.shape) for t in self.params] for _ in "mv")
        self.grads = [E(*t.shape, dtype=BF) for t in self.params]  # what the step takes
        self.dW = [E(DIM, DIM, dtype=BF) for _ in range(BLOCKS)]
        self.x, self.res = rnd(ROWS, DIM).to(BF), rnd(ROWS, DIM)
        self.target = rnd(ROWS, DIM)
        self.h = [E(ROWS, DIM) for _ in range(BLOCKS)]
        self.rstd = [E(ROWS) for _ in range(BLOCKS)]
        self.codes = [E(ROWS, DIM, dtype=torch.uint8) for _ in range(BLOCKS)]
        self.scales = [E(ROWS, -(-DIM // 32), dtype=torch.uint8) for _ in range(BLOCKS)]
        need = max(LC.lc_norm_backward_workspace(ROWS, DIM), LC.lc_linear_wgrad_workspace(ROWS, DIM, DIM),
                   LC.lc_orthogonalize_workspace(BLOCKS, DIM, DIM, LC.LC_DT_BF16))
        self.ws, self.need = torch.zeros(need, dtype=torch.uint8, device="cuda"), need
        segs = [LC.Segment(i // 2, p.numel(), p.data_ptr(), None, q.data_ptr(), m.data_ptr(), v.data_ptr())
                for i, (p, q, m, v) in enumerate(zip(self.params, self.master, self.m, self.v))]
        self.layout = LC.LayoutDesc(segs, BLOCKS, LC.LC_DT_BF16, True, LC.LC_MODE_ACCUM, [0.0] * BLOCKS, 1 << 20, stream=stream())
        self.ctx = LC.lc_init_layout(self.layout)
        self.t = 0

    def close(self):
        LC.lc_destroy(self.ctx)

    def norm(self, i):
        return LC.norm_params(LC.LC_NORM_RMS, self.w[i].data_ptr(), 0, LC.LC_DT_BF16, 1e-5)

    def gradients(self):
        x, h = self.x, self.res
        self.xs = []
        for i in range(BLOCKS):
            y8 = LC.saved_act(self.codes[i].data_ptr(), self.scales[i].data_ptr(), ROWS, DIM)
            y = torch.empty(ROWS, DIM, dtype=BF, device="cuda")
            LC.lc_residual_norm_forward(self.norm(i), M(x), M(h), M(self.h[i]), M(y), rstd=self.rstd[i].data_ptr(), y_saved=y8,
                                        stream=stream())
            self.xs.append(x)
            x, h = (y.float() @ self.W[i].float().t()).to(BF), self.h[i]
        dh = (h + x.float() - self.target) / (ROWS * DIM)
        for i in reversed(range(BLOCKS)):
            dz = dh.to(BF)
            y8 = LC.saved_act(self.codes[i].data_ptr(), self.scales[i].data_ptr(), ROWS, DIM)
            LC.lc_linear_wgrad(M(dz), y8, M(self.dW[i]), self.ws.data_ptr(), self.need, stream=stream())
            dy = (dz.float() @ self.W[i].float()).to(BF)
            dres = torch.empty(ROWS, DIM, device="cuda")
            LC.lc_residual_norm_backward(self.norm(i), M(dy), M(dh), self.rstd[i].data_ptr(), None, M(dres), self.grads[2 * i + 1].data_ptr(),
                                         0, LC.LC_DT_BF16, self.ws.data_ptr(), self.need, h=M(self.h[i]), stream=stream())
            dh = dres
        self.dres = dh

    def step(self):
        self.gradients()
        LC.lc_orthogonalize(LC.orthogonalize_params(5, None, 0.95, True, 1e-7, 0.2 * DIM ** 0.5), [M(t) for t in self.dW],
                            [M(t) for t in self.grads[::2]], self.ws.data_ptr(), self.need, momenta=[M(t) for t in self.m[::2]],
                            stream=stream())
        self.t += 1
        LC.lc_muon_step_score(self.ctx, self.t, [t.data_ptr() for t in self.grads], LC.LC_DT_BF16, [1, 0] * BLOCKS, lr=1e-3, beta1=0.9,
                              beta2=0.95, eps=1e-8, weight_decay=0.1, ortho_lr=2e-3, ortho_weight_decay=0.05, adam_step=self.t,
                              decay_mask=[1, 0] * BLOCKS)

    def state(self):
        return self.params + self.master + self.m + self.v


def test_gradients_are_those_of_the_loss():
    """Against autograd in 64 bits.  Each block's values pass a handful of bf16 roundings of 2^-9 of their root mean square on
    their way (y, x, dz, dy, the result), y in 8 bits one of 2^-4 / sqrt(3) at most in W's gradient, all of either sign and
    of independent elements: in norm, twelve of the former behind three blocks, each raised by the products by no more than |W|
    (2.4) a block, and one of the latter."""
    p = Program(3)
    try:
        p.gradients()
        W = [t.double().requires_grad_() for t in p.W]
        w = [t.double().requires_grad_() for t in p.w]
        res = p.res.double().requires_grad_()
        x, h = p.x.double(), res
        for i in range(BLOCKS):
            h = x + h
            x = (h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-5) * w[i]) @ W[i].t()
        (0.5 * (h + x - p.target.double()).square().mean()).backward()
        off = lambda a, b: ((a.double() - b).norm() / b.norm()).item()  # noqa: E731
        rounding = 12 * 2.0 ** -9
        assert off(p.dres, res.grad) <= rounding
        for i in range(BLOCKS):
            assert off(p.dW[i], W[i].grad) <= rounding + 2.0 ** -4
            assert off(p.grads[2 * i + 1], w[i].grad) <= rounding * 2
    finally:
        p.close()


def test_a_run_goes_on_from_its_checkpoint():
    """Steps 3 and 4 from the restored state give every bit that they gave the first time."""
    p = Program(4)
    try:
        _, rec = LC.lc_query_layout(p.layout)
        staging = torch.zeros(sum(int(r) for r in rec), dtype=torch.uint8, device="cuda")
        start = [t.clone() for t in p.state()]
        p.step()
        p.step()
        mask, _ = LC.lc_select(p.ctx, 2, 1.0, BLOCKS)
        assert mask.all()
        LC.lc_pack_selected(p.ctx, staging.data_ptr(), staging.numel())
        p.step()
        p.step()
        torch.cuda.synchronize()
        want = [t.clone() for t in p.state()]
        assert all(not torch.equal(a, b) for a, b in zip(start[:2 * BLOCKS], want)) and all(torch.isfinite(t).all() for t in want)
        moved = [t.view(-1)[0].item() for t in p.v[::2]]
        assert moved == [0.0] * BLOCKS  # an orthogonalised matrix has no second moment
        for t in p.state():
            t.fill_(7)
        LC.lc_restore_composite(p.ctx, [{"step": 2, "mask": mask, "payload": staging.data_ptr(), "payload_bytes": staging.numel()}], 2,
                                BLOCKS)
        p.t = 2
        p.step()
        p.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p.state(), want))
    finally:
        p.close()


def test_updates_are_near_orthogonal():
    """What the mixed step takes of a matrix has singular values of one size: within 0.6 and 1.25 of the scale, but for the few
    that the gradient hardly has (five steps raise one by 3.44^5 at most, so those above 0.7 / 480 of u's norm get there)."""
    p = Program(5)
    try:
        p.step()
        torch.cuda.synchronize()
        for dW, o, buf in zip(p.dW, p.grads[::2], p.m[::2]):
            assert torch.equal(buf, dW.float())  # from a momentum of zeros
            sv = torch.linalg.svdvals(o.double().cpu()) / (0.2 * DIM ** 0.5)
            there = torch.linalg.svdvals(dW.double().cpu()) / dW.double().norm().item()
            assert sv.max() < 1.25 and sv[: int((there > 0.01).sum())].min() > 0.6
    finally:
        p.close()


def test_grids_capped_at_forty_blocks():
    """The same files on the build whose launches have forty blocks at most: blocks that take several tiles, rows or chunks."""
    if not os.path.exists(GRID_CAPPED_LIB):
        pytest.skip("the grid-capped library is built by __graft_entry__.build()")
    if os.environ.get("LAYERCHECK_LIB"):
        pytest.skip("runs in the parent only")
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "-m", "gpu", "-k", "not beyond_32 and not streams",
                        *(os.path.join("tests", f) for f in ("test_residual_norm_gpu.py", "test_orthogonalize_gpu.py", "test_muon_gpu.py",
                                                             "test_training_block_gpu.py"))],
                       env=dict(os.environ, LAYERCHECK_LIB=GRID_CAPPED_LIB), cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
