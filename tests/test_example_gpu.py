"""The example of a training step: its gradients against the formulas in 64 bits, and that it learns."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_gradients_of_a_step():
    import train_step as E
    m = E.Model(vocab=96, dim=160, tokens=300)
    try:
        m.w[1].copy_(1 + 0.2 * torch.randn(1, 160, device="cuda"))
        tokens, target = E.batch(m, 1)
        logits = m.forward(tokens)
        _, dz = m.loss(logits, target)
        m.backward(tokens, dz)
        # a bf16 rounding of each array on the way, 8-bit rows (2^-4 an element at most, averaged over many) in place of n
        h = m.w[0].double()[tokens] * m.scale
        rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + E.EPS)
        n, w, d = h * rstd, m.w[1].double(), dz.double()
        dy = d @ m.w[2].double()
        g = dy * w
        dh = rstd * (g - n * (g * n).mean(1, keepdim=True))
        want = [torch.zeros(96, 160, dtype=torch.float64, device="cuda").index_add_(0, tokens, dh) * m.scale,
                (dy * n).sum(0, keepdim=True), d.t() @ (n * w)]
        for got, ref in zip(m.grad, want):
            assert ((got.double() - ref).norm() / ref.norm()).item() <= 2.0 ** -4
    finally:
        m.close()


def test_it_learns():
    import train_step as E
    assert E.main(40) < 0.5 * math.log(512)
