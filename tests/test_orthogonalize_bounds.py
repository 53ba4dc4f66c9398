"""The bound on the largest singular value that the orthogonalised update reckons with, from which calls it refuses (CPU: no call
here enqueues anything).  X is held times a power of two that the bound allows: one that is too small lets fp16 overflow."""
import os

import numpy as np
import pytest

from paper_2609_27193_amd import layercheck as LC
from tests.test_more_operators_abi import ortho
from tests.test_operators_abi import refused

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "layercheck.h")


ROUNDINGS = 1.005


def largest(coefs):
    """What the steps let it grow to, by a dense scan of each polynomial: they start from 1, and a step adds 0.5% for roundings."""
    top = 1.0
    for a, b, c in coefs:
        s = np.linspace(0.0, top, 200001)
        top = ROUNDINGS * np.abs(s * (a + s * s * (b + s * s * c))).max()
    return top


BOUNDS = [[(3.4445, -4.775, 2.0315)] * 5, [(1.5, -0.5, 0.0)] * 9, [(2.0, -1.5, 0.5)] * 4, [(0.0, 3.0, -2.0)], [(1.0, 0.0, -1.0)] * 2,
          [(-1.0, 0.0, 0.0)], [(1.6, -2.0, 0.7)] * 3, [(0.0, 0.0, 1.0)], [(1e-3, -2e-3, 1e-3)]]
# c of what is left of a subtraction, or of a fit: the steps end near the polynomial's zero, with its largest value inside
BOUNDS += [[(1.698, 0.0, 0.0), (1.5, -0.5, c)] for c in (1e-18, -1e-18, 1e-12, -1e-12, 1e-9, 1e-6, 5e-324, 1e-300, 0.0)]
BOUNDS += [[(0.98, 0.0, 0.0), (1.0, b, -1.0)] for b in (1e-18, -1e-18, 1e-9, 0.0)]
BOUNDS += [[(0.98, 0.0, 0.0), (a, 1.0, -1.0)] for a in (1e-18, -1e-18, 1e-9, 0.0)]


@pytest.mark.parametrize("coefs", BOUNDS)
def test_ortho_bound_is_the_largest_value_of_the_steps(coefs):
    """One step more, of a factor alone, that brings the bound just below or above the most and the least that are taken."""
    for edge, inside in ((2.0 ** 30, 0.999), (2.0 ** -30, 1.001)):
        k = edge / (ROUNDINGS * largest(coefs))
        refused(ortho, prm=LC.orthogonalize_params(len(coefs) + 1, coefs + [(k * inside, 0.0, 0.0)]), size=0, says="workspace",
                code=LC.LC_ERR_CAPACITY)  # the coefficients are taken
        refused(ortho, prm=LC.orthogonalize_params(len(coefs) + 1, coefs + [(k / inside, 0.0, 0.0)]), size=0, says="singular")


# Each step's polynomial turns upwards right behind the range that the one before leaves: 1.99, 1.97, 1.87, 1.56, 1.13, 1.
SHARP = [(8.2, -22.9, 16.5), (4.07, -2.87, 0.522), (3.92, -2.83, 0.53), (3.29, -2.42, 0.49), (2.28, -1.62, 0.40), (1.87, -1.23, 0.36),
         (1.875, -1.25, 0.375)]


def test_steps_that_need_their_range_are_taken():
    """The largest singular value stays below 2 in exact arithmetic; what is added for roundings must not run away with it."""
    assert largest(SHARP) < 1.1
    for n in range(1, len(SHARP) + 1):
        refused(ortho, prm=LC.orthogonalize_params(n, SHARP[:n]), size=0, says="workspace", code=LC.LC_ERR_CAPACITY)


GIB = 1 << 30


@pytest.mark.parametrize("rows,cols", [(256, 65536), (65536, 512), (1024, 65536), (2000, 60000), (300, 40000), (4096, 65536)])
@pytest.mark.parametrize("dtype", [LC.LC_DT_BF16, LC.LC_DT_F32], ids=["bf16", "f32"])
def test_workspace_of_many_long_matrices(rows, cols, dtype):
    """X goes from one buffer to another, each of 4 bytes an element in padded sides, beside A and B of 4 or 2: as many matrices as
    take 4 GiB of these are worked on at once, or one; the rest of the workspace are sums and parts of sums."""
    m, n = (-(-x // 64) * 64 for x in sorted((rows, cols)))
    each = 8 * m * n + 8 * m * m
    alone = LC.lc_orthogonalize_workspace(1, rows, cols, dtype)
    needs = [LC.lc_orthogonalize_workspace(count, rows, cols, dtype) for count in (1, 2, 5, 8, 15, 16, 17, 40, 64)]
    assert max(needs) <= max(4 * GIB, each) + 256 * (1 << 20)
    assert needs == sorted(needs) and needs[0] == alone


def test_momentum_is_checked_without_momenta_too():
    """As the header says: it lies in [0, 1) in any call."""
    for bad in (1.0, -0.1, np.nan):
        refused(ortho, prm=LC.orthogonalize_params(5, momentum=bad), says="momentum")
    for good in (0.0, 0.95):
        refused(ortho, prm=LC.orthogonalize_params(5, momentum=good), size=0, says="workspace", code=LC.LC_ERR_CAPACITY)
    assert "mu, in [0, 1) in any call" in open(HEADER).read()
