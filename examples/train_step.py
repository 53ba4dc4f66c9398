"""A training loop whose gradients and optimizer steps all come from the library: one process, one GPU.

The model is the smallest that has every operator: a scaled embedding, an RMS norm and a linear head, trained to say the
next token of a made-up language (each token has one successor).  A step is

  lc_embedding_forward     h = scale * E[token]
  lc_norm_forward          y = RMSNorm(h); the normalised rows stay in 8 bits, h and y are not kept
  (torch)                  logits = y W^T, softmax cross entropy and its gradient dz
  lc_linear_wgrad          dW from dz and the kept rows, the norm's weight applied on the way
  lc_norm_backward         dh and the norm's gradient from the same rows
  lc_embedding_backward    dE by sorted tokens
  lc_adamw_step_score      AdamW on the three layers, with their drift
  lc_select, lc_pack_selected   the layers whose drift is due, packed for the checkpoint

Run: ``python examples/train_step.py``
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2609_27193_amd import layercheck as LC  # noqa: E402

BF, F32 = LC.LC_DT_BF16, LC.LC_DT_F32
EPS = 1e-5


def view(t):
    """The library's view of a two-dimensional tensor, whose rows lie apart and whose columns lie side by side."""
    if t.dim() != 2 or t.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError(f"{t.dim()} dimensions of {t.dtype}: a matrix in bf16 or fp32 is needed")
    if (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
        raise ValueError(f"strides of {t.stride()} for {tuple(t.shape)}: rows of neighbouring columns are needed")
    return LC.matrix(t.data_ptr(), t.shape[0], t.shape[1], BF if t.dtype == torch.bfloat16 else F32, t.stride(0))


class Model:
    LAYERS = ("embed_tokens", "norm", "lm_head")

    def __init__(self, vocab=512, dim=256, tokens=4096, seed=0, k0=0.02, s_max=10):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.dim, self.n = vocab, dim, tokens
        self.scale = dim ** 0.5
        self.stream = torch.cuda.current_stream().cuda_stream
        shapes = [(vocab, dim), (1, dim), (vocab, dim)]
        init = [torch.randn(s, generator=g, device="cuda") * 0.02 for s in shapes]
        init[1].fill_(1)
        # per layer: weights in bf16, master, moments and gradient
        self.master = init
        self.w = [p.bfloat16() for p in init]
        self.m, self.v = ([torch.zeros_like(p) for p in init] for _ in "mv")
        self.grad = [torch.empty_like(w) for w in self.w]
        segs = [LC.Segment(i, w.numel(), w.data_ptr(), None, p.data_ptr(), m.data_ptr(), v.data_ptr())
                for i, (w, p, m, v) in enumerate(zip(self.w, self.master, self.m, self.v))]
        layout = LC.LayoutDesc(segs, 3, BF, True, LC.LC_MODE_ACCUM, [k0] * 3, s_max, stream=self.stream)
        self.ctx = LC.lc_init_layout(layout)
        self.staging = torch.empty(sum(LC.lc_record_bytes(self.ctx, i) for i in range(3)), dtype=torch.uint8, device="cuda")
        # activations, and what the backward pass has of them
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.h, self.y, self.dh = (torch.empty(tokens, dim, **bf) for _ in range(3))
        self.rstd = torch.empty(tokens, device="cuda")
        self.codes = torch.empty(tokens, dim, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(tokens, -(-dim // LC.ACT_BLOCK), dtype=torch.uint8, device="cuda")
        self.kept = LC.saved_act(self.codes.data_ptr(), self.scales.data_ptr(), tokens, dim)
        self.norm = LC.norm_params(LC.LC_NORM_RMS, self.w[1].data_ptr(), 0, BF, EPS)
        need = max(LC.lc_embedding_backward_workspace(tokens, dim), LC.lc_norm_backward_workspace(tokens, dim),
                   LC.lc_linear_wgrad_workspace(tokens, vocab, dim))
        self.space = torch.empty(need, dtype=torch.uint8, device="cuda")
        LC.lc_pack_selected(self.ctx, self.staging.data_ptr(), self.staging.numel())  # the base version

    def forward(self, tokens):
        LC.lc_embedding_forward(view(self.w[0]), tokens.data_ptr(), LC.LC_IT_I64, self.n, view(self.h), scale=self.scale,
                                stream=self.stream)
        LC.lc_norm_forward(self.norm, view(self.h), view(self.y), rstd=self.rstd.data_ptr(), saved=self.kept,
                           stream=self.stream)
        return torch.mm(self.y, self.w[2].t()).float()

    def loss(self, logits, target):
        """Mean cross entropy, and its gradient."""
        logp = torch.log_softmax(logits, 1)
        dz = logp.exp()
        dz[torch.arange(self.n, device="cuda"), target] -= 1
        return -logp[torch.arange(self.n, device="cuda"), target].mean(), (dz / self.n).bfloat16()

    def backward(self, tokens, dz):
        a, size, st = self.space.data_ptr(), self.space.numel(), self.stream
        LC.lc_linear_wgrad(view(dz), self.kept, view(self.grad[2]), a, size, col_scale=self.w[1].data_ptr(), param_dtype=BF,
                           stream=st)
        dy = torch.mm(dz, self.w[2])
        LC.lc_norm_backward(self.norm, view(dy), self.rstd.data_ptr(), view(self.dh), self.grad[1].data_ptr(), None, BF, a,
                            size, saved=self.kept, stream=st)
        LC.lc_embedding_backward(view(self.dh), tokens.data_ptr(), LC.LC_IT_I64, self.n, view(self.grad[0]), a, size,
                                 scale=self.scale, stream=st)

    def step(self, t, tokens, target, lr=1e-2):
        """One training step and its checkpoint decision: (loss, names of the layers persisted)."""
        loss, dz = self.loss(self.forward(tokens), target)
        self.backward(tokens, dz)
        LC.lc_adamw_step_score(self.ctx, t, [g.data_ptr() for g in self.grad], BF, lr, 0.9, 0.95, 1e-8, 0.0, t)
        mask, _ = LC.lc_select(self.ctx, t, 1.0, 3)
        if mask.any():
            LC.lc_pack_selected(self.ctx, self.staging.data_ptr(), self.staging.numel())
        return loss.item(), [name for name, on in zip(self.LAYERS, mask) if on]

    def close(self):
        LC.lc_destroy(self.ctx)


def batch(model, seed):
    """Tokens of the made-up language and the ones that follow them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    tokens = torch.randint(0, model.vocab, (model.n,), generator=g, device="cuda")
    return tokens, (tokens * 7 + 3) % model.vocab


def main(steps=40):
    model = Model()
    try:
        for t in range(1, steps + 1):
            loss, kept = model.step(t, *batch(model, t))
            if t % 5 == 0 or t == 1:
                print("step %3d  loss %.4f  persisted: %s" % (t, loss, ", ".join(kept) or "none"), flush=True)
        held = model.codes.numel() + model.scales.numel()
        print("activations held for the backward pass: %d bytes in 8 bits, %d as the norm's input and output in bf16"
              % (held, 2 * 2 * model.h.numel()))
        return loss
    finally:
        model.close()


if __name__ == "__main__":
    main()
