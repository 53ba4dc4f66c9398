"""The forms in perf/operators.py, plain and the library's, against its results in 64 bits, at its small cases and drawn ones.

This holds the formulas together, not the roundings: an array's error is measured in its norm.  A bf16 result is off by 2^-8 at
most, an element in 8 bits by 2^-4.  A sum of n fp32 addends is off by n 2^-24 of their magnitudes' sum at most, which for
addends of either sign is some sqrt(n) of the sum itself: below 2^-10 for 600 rows."""
import random

import pytest
import torch

import perf.operators as P

pytestmark = pytest.mark.gpu

ROWS = 600
BOUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -10}


def cases():
    out = [c for c in P.listed() if c["rows"] <= ROWS]
    rng = random.Random(7)
    count = dict.fromkeys(P.OPS, 0)
    while min(count.values()) < 4:
        c = P.draw(rng)
        if c["rows"] <= ROWS and count[c["op"]] < 4 and c.get("vocab", 0) * c.get("dim", 0) <= 1 << 26:
            count[c["op"]] += 1
            out.append(c | {"name": f"{c['op']}_{count[c['op']]}"})
    return out


def arrays(result):
    return result if isinstance(result, dict) else {"": result}


@pytest.mark.parametrize("case", cases(), ids=lambda c: c["name"])
@pytest.mark.parametrize("own", [False, True], ids=["plain", "library"])
def test_forms_agree_with_the_definition(case, own, monkeypatch):
    monkeypatch.setattr(P, "own", own)
    got, want = arrays(P.run(P.prepare(case, 3))), arrays(P.exact(case, 3))
    assert got.keys() == want.keys()
    for name, g in got.items():
        bound = 2.0 ** -4 if name == "kept" else BOUND[g.dtype]
        assert g.shape == want[name].shape
        assert ((g.double() - want[name]).norm() <= bound * want[name].norm()).item(), (name, (g.double() - want[name]).norm() / want[name].norm())
