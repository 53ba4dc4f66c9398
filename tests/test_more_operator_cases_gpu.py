"""The forms in perf/more_operators.py, plain and the library's, against its results in 64 bits, at its small cases and drawn ones.

This holds the formulas together, not the roundings: an array's error is measured in its norm.  A bf16 result is off by 2^-8 at
most, an element in 8 bits by 2^-4.  A sum of n fp32 addends is off by n 2^-24 of their magnitudes' sum at most, which for
addends of either sign is some sqrt(n) of the sum itself: below 2^-10 for 600 rows.

The Newton-Schulz steps start from |X| = 1 and end with m singular values of some 0.7 or more, sqrt(m) / 2 of norm at least,
and raise what a rounding left in a singular direction by at most the first coefficient each, a^5 in all and a^5 / (1 - 1 / a)
with the roundings of the later steps.  A plane of 11 bits is off by 2^-12 of its norm: 2^-12 a^5 sqrt(m) 2 (1 + 2 / (a - 1)) / m
covers X's own (X, A and B each bring one, and a result whose values never reach 0.7 is a^5 |X| itself and off by no more)."""
import random

import pytest
import torch

import perf.more_operators as P

pytestmark = pytest.mark.gpu

MOST = 1 << 20
BOUND = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -10}


def small(c):
    if c["op"] == "muon":
        return sum(k for _, k, _, _ in P._tensors(c)) <= 1 << 23
    return c["rows"] * c["cols" if c["op"] == "ortho" else "dim"] * c.get("n", 1) <= MOST and c["rows"] <= 600


def cases():
    out = [c for c in P.listed() if small(c)]
    rng = random.Random(7)
    count = dict.fromkeys(P.OPS, 0)
    while min(count.values()) < 6:
        c = P.draw(rng)
        if small(c) and count[c["op"]] < 6:
            count[c["op"]] += 1
            out.append(c | {"name": f"{c['op']}_{count[c['op']]}"})
    return out


def arrays(result, name=""):
    if result is None:
        return {}
    if isinstance(result, (dict, list)):
        items = result.items() if isinstance(result, dict) else enumerate(result)
        return {k: v for i, r in items for k, v in arrays(r, f"{name}/{i}").items()}
    return {name: torch.as_tensor(result, device="cuda")}


def steps_bound(c):
    a, m = P.COEFS[c["coefs"]][0], min(c["rows"], c["cols"])
    h = 2.0 ** -12 if c["out"] == "bf16" else 2.0 ** -21
    return h * a ** P.STEPS * 2 * (1 + 2 / (a - 1)) / m ** 0.5


@pytest.mark.parametrize("case", cases(), ids=lambda c: c["name"])
@pytest.mark.parametrize("own", [False, True], ids=["plain", "library"])
def test_forms_agree_with_the_definition(case, own, monkeypatch):
    monkeypatch.setattr(P, "own", own)
    got, want = arrays(P.run(P.prepare(case, 3))), arrays(P.exact(case, 3))
    assert got.keys() == want.keys()
    for name, g in got.items():
        bound = 2.0 ** -4 if name in ("/kept", "/y8") else BOUND[g.dtype]
        if name.startswith("/out"):
            bound += steps_bound(case)
        off, size = (g.double() - want[name].double()).norm(), want[name].double().norm()
        assert g.shape == want[name].shape
        assert (off <= bound * size).item(), (name, off / size)
