"""The mixed optimizer step: parameters, moments and weights bit for bit against the same fp32 operations in numpy, one rounding
each, and the drift against its definition in 64 bits.

The kernel adds four fp32 terms of the drift pairwise before it goes on in 64 bits: two roundings of 2^-24 of a positive sum, in
both of u's sums."""
import numpy as np
import pytest
import torch

from paper_2609_27193_amd import layercheck as LC
from tests.test_operators_gpu import stream

pytestmark = pytest.mark.gpu

F = np.float32
BF16 = torch.bfloat16
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, ortho_lr=0.02, ortho_weight_decay=0.05)
EPS_W = 1e-8


class Model:
    """Layers of segments (numel, decay, ortho); every array starts `shift` elements into a buffer of its own."""

    def __init__(self, layers, dtype, master, grad, shift=0, seed=0, k0=1e6):
        g = torch.Generator().manual_seed(seed)
        dt = BF16 if dtype == "bf16" else torch.float32
        self.gt = BF16 if grad == "bf16" else torch.float32
        self.segs = [(i, n, d, o) for i, layer in enumerate(layers) for n, d, o in layer]
        self.n_layers, self.master = len(layers), master

        def place(v, dtype):
            t = torch.zeros(v.numel() + shift, dtype=dtype, device="cuda")
            t[shift:] = v
            return t[shift:]

        rnd = lambda n, s: torch.randn(n, generator=g) * s  # noqa: E731
        self.p = [rnd(n, 0.02) for _, n, _, _ in self.segs]
        self.w = [place(p, dt) for p in self.p]
        self.mst = [place(p, torch.float32) if master else None for p in self.p]
        self.m = [place(rnd(n, 1e-3), torch.float32) for _, n, _, _ in self.segs]
        self.v = [place(rnd(n, 1e-6).abs(), torch.float32) for _, n, _, _ in self.segs]
        self.grad = [place(rnd(n, 0.2 if o else 1e-3), self.gt) for _, n, _, o in self.segs]
        at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        segs = [LC.Segment(i, n, at(w), None, at(q), at(m), at(v))
                for (i, n, _, _), w, q, m, v in zip(self.segs, self.w, self.mst, self.m, self.v)]
        self.layout = LC.LayoutDesc(segs, self.n_layers, LC.LC_DT_BF16 if dtype == "bf16" else LC.LC_DT_F32, master, LC.LC_MODE_ACCUM,
                                    [k0] * self.n_layers, 1 << 20, eps_w=EPS_W, stream=stream())
        self.ctx = LC.lc_init_layout(self.layout)
        self.decay, self.ortho = [d for _, _, d, _ in self.segs], [o for _, _, _, o in self.segs]
        self.addresses = [t.data_ptr() for t in self.grad]
        self.gdt = LC.LC_DT_BF16 if grad == "bf16" else LC.LC_DT_F32

    def close(self):
        LC.lc_destroy(self.ctx)

    def host(self):
        f = lambda ts: [None if t is None else t.float().cpu().numpy() for t in ts]  # noqa: E731
        return dict(p=f(self.mst if self.master else self.w), w=f(self.w), m=f(self.m), v=f(self.v), g=f(self.grad))

    def step(self, t, ortho=None, decay=None, **kw):
        LC.lc_muon_step_score(self.ctx, t, self.addresses, self.gdt, self.ortho if ortho is None else ortho, adam_step=t,
                              decay_mask=self.decay if decay is None else decay, **{**HYPER, **kw})


def bf16_of(x):
    return torch.from_numpy(x).to(BF16).float().numpy()


def stepped(s, segs, t, bf16_weights, hy=HYPER):
    """One step in fp32, an operation at a time."""
    b1, b2 = F(hy["beta1"]), F(hy["beta2"])
    omb1, omb2 = F(1.0 - hy["beta1"]), F(1.0 - hy["beta2"])
    c1, c2 = F(1.0 / (1.0 - hy["beta1"] ** t)), F(1.0 / (1.0 - hy["beta2"] ** t))
    out = dict(p=[], w=[], m=[], v=[])
    for i, (_, _, d, o) in enumerate(segs):
        p, m, v, g = s["p"][i], s["m"][i], s["v"][i], s["g"][i]
        if o:
            lr, dec, upd = F(hy["ortho_lr"]), F(1.0 - hy["ortho_lr"] * hy["ortho_weight_decay"]), g
        else:
            lr, dec = F(hy["lr"]), F(1.0 - hy["lr"] * hy["weight_decay"])
            m = b1 * m + omb1 * g
            v = b2 * v + omb2 * (g * g)
            upd = (m * c1) / (np.sqrt(v * c2) + F(hy["eps"]))
        q = (p * dec if d else p) - lr * upd
        out["p"].append(q)
        out["w"].append(bf16_of(q) if bf16_weights else q)
        out["m"].append(m)
        out["v"].append(v)
    return out


def drift(segs, n_layers, before, after):
    u = []
    for layer in range(n_layers):
        a = np.concatenate([before[i].astype(np.float64) for i, s in enumerate(segs) if s[0] == layer])
        b = np.concatenate([after[i].astype(np.float64) for i, s in enumerate(segs) if s[0] == layer])
        d = np.abs((b - a).astype(F).astype(np.float64))  # one fp32 subtraction
        u.append(d.mean() / (np.abs(a).mean() + EPS_W))
    return np.array(u)


LAYERS = {"small": [[(40, 1, 0)], [(17, 1, 1), (5, 0, 0), (33, 0, 1)], [(1, 0, 0)], [(3, 1, 1)]],
          "chunks": [[(9000, 1, 0), (4096, 0, 1)], [(8192, 1, 1), (12288, 1, 0), (20001, 1, 1)], [(777, 0, 0)]],
          "many": [[(10 + i, i % 2, (i // 2) % 2)] for i in range(300)]}  # more segments than the kernel's arguments hold


@pytest.mark.parametrize("layers", LAYERS)
@pytest.mark.parametrize("dtype,master", [("bf16", True), ("bf16", False), ("f32", False), ("f32", True)])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [0, 3])
def test_steps(layers, dtype, master, grad, shift):
    x = Model(LAYERS[layers], dtype, master, grad, shift)
    try:
        delta = np.zeros(x.n_layers)
        for t in (1, 2, 3):
            before = x.host()
            want = stepped(before, x.segs, t, dtype == "bf16")
            x.step(t)
            u, d, _ = LC.lc_read_state(x.ctx, x.n_layers)
            got = x.host()
            for name in ("p", "w", "m", "v") if master or dtype == "f32" else ("w", "m", "v"):
                for i, (a, b) in enumerate(zip(got[name], want[name])):
                    assert np.array_equal(a, b), (name, i, t)
            ref = drift(x.segs, x.n_layers, before["p"], want["p"])
            assert np.all(np.abs(u - ref) <= 6 * 2.0 ** -24 * ref), t
            delta += u
            assert np.allclose(d, delta, rtol=1e-12)
    finally:
        x.close()


@pytest.mark.parametrize("dtype,master", [("bf16", True), ("f32", False)])
def test_masks_of_one_kind_are_the_other_steps(dtype, master):
    """An ortho_mask of zeros gives lc_adamw_step_score's bits, one of ones lc_sgd_step_score's, and leaves the moments."""
    for ortho in (0, 1):
        a, b = (Model(LAYERS["chunks"], dtype, master, "f32", 1) for _ in "ab")
        try:
            a.step(1, [ortho] * len(a.segs))
            if ortho:
                LC.lc_sgd_step_score(b.ctx, 1, b.addresses, b.gdt, HYPER["ortho_lr"], HYPER["ortho_weight_decay"], b.decay)
            else:
                LC.lc_adamw_step_score(b.ctx, 1, b.addresses, b.gdt, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"],
                                       HYPER["weight_decay"], 1, b.decay)
            ha, hb = a.host(), b.host()
            for name in ("p", "w", "m", "v"):
                assert all(np.array_equal(s, t) for s, t in zip(ha[name], hb[name])), name
            assert np.array_equal(LC.lc_read_state(a.ctx, a.n_layers)[0], LC.lc_read_state(b.ctx, b.n_layers)[0])
        finally:
            a.close()
            b.close()


def test_refusals_change_nothing():
    x = Model(LAYERS["small"], "bf16", True, "bf16")
    try:
        before = x.host()
        n = len(x.segs)
        for bad, says in [(dict(ortho=[2] * n), "ortho_mask"), (dict(decay=[3] * n), "decay_mask"), (dict(ortho_lr=-1.0), "ortho_lr"),
                          (dict(ortho_lr=float("nan")), "ortho_lr"), (dict(ortho_weight_decay=float("inf")), "ortho_weight_decay"),
                          (dict(ortho_weight_decay=-0.1), "ortho_weight_decay"), (dict(lr=-1.0), "lr"), (dict(beta1=1.0), "betas"),
                          (dict(eps=0.0), "eps")]:
            with pytest.raises(LC.LCError) as e:
                x.step(1, **bad)
            assert e.value.code == LC.LC_ERR_INVALID_ARG and says in str(e.value), bad
        lib = LC.load_library()
        prm = LC.lc_muon_params(LC.lc_adamw_params(1e-3, 0.9, 0.95, 1e-8, 0, 1), 1e-3, 0)
        grads = LC._addresses(x.addresses)
        assert lib.lc_muon_step_score(x.ctx, 1, grads, x.gdt, None, None, prm) == LC.LC_ERR_INVALID_ARG
        assert lib.lc_muon_step_score(x.ctx, 1, None, x.gdt, LC._mask(x.ortho)[0], None, prm) == LC.LC_ERR_INVALID_ARG
        assert lib.lc_muon_step_score(x.ctx, 1, grads, x.gdt, LC._mask(x.ortho)[0], None, None) == LC.LC_ERR_INVALID_ARG
        x.step(1)
        with pytest.raises(LC.LCError) as e:
            x.step(1)  # the step does not increase
        assert e.value.code == LC.LC_ERR_BAD_STATE
        with pytest.raises(LC.LCError) as e:
            LC.lc_score_layers(x.ctx, 2)  # the shadow is stale
        assert e.value.code == LC.LC_ERR_BAD_STATE
        want = stepped(before, x.segs, 1, True)
        assert all(np.array_equal(a, b) for a, b in zip(x.host()["w"], want["w"]))
    finally:
        x.close()


def test_no_moments_no_mixed_step():
    w = torch.zeros(64, device="cuda")
    layout = LC.LayoutDesc([LC.Segment(0, 64, w.data_ptr(), None, None, None, None)], 1, LC.LC_DT_F32, False, LC.LC_MODE_ACCUM,
                           [1.0], 10, stream=stream())
    ctx = LC.lc_init_layout(layout)
    try:
        with pytest.raises(LC.LCError) as e:
            LC.lc_muon_step_score(ctx, 1, [w.data_ptr()], LC.LC_DT_F32, [1], adam_step=1, **HYPER)
        assert e.value.code == LC.LC_ERR_BAD_STATE and "moments" in str(e.value)
    finally:
        LC.lc_destroy(ctx)


def test_decision_and_recovery():
    """The step, the decision, the pack and a restore: the momentum of an orthogonalised matrix comes back with its layer."""
    x = Model(LAYERS["chunks"], "bf16", True, "bf16", k0=0.0)
    try:
        _, rec = LC.lc_query_layout(x.layout)
        staging = torch.zeros(sum(int(r) for r in rec), dtype=torch.uint8, device="cuda")
        x.step(1)
        for m, (_, _, _, o) in zip(x.m, x.segs):
            if o:
                m.mul_(0.95).add_(0.1)  # as lc_orthogonalize leaves it
        mask, _ = LC.lc_select(x.ctx, 1, 1.0, x.n_layers)
        assert mask.all()
        with pytest.raises(LC.LCError) as e:
            x.step(2)  # the selection is not packed yet
        assert e.value.code == LC.LC_ERR_BAD_STATE
        LC.lc_pack_selected(x.ctx, staging.data_ptr(), staging.numel())
        torch.cuda.synchronize()
        kept = x.host()
        for t in x.w + x.mst + x.m + x.v:
            t.fill_(5)
        LC.lc_restore_composite(x.ctx, [{"step": 1, "mask": mask, "payload": staging.data_ptr(), "payload_bytes": staging.numel()}], 1,
                                x.n_layers)
        back = x.host()
        for name in ("p", "w", "m", "v"):
            assert all(np.array_equal(a, b) for a, b in zip(kept[name], back[name])), name
        x.step(2)
        want = stepped(kept, x.segs, 2, True)
        assert all(np.array_equal(a, b) for a, b in zip(x.host()["p"], want["p"]))
    finally:
        x.close()
