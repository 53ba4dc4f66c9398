"""The example's view of a tensor takes what the library can read, and refuses the rest (CPU)."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_views_of_tensors():
    import train_step as E
    t = torch.zeros(6, 8, dtype=torch.bfloat16)
    for part in (t, t[1:4], t[:, 2:5], t[::2], t[3:4, 1:]):
        m = E.view(part)
        assert (m.data, m.rows, m.cols, m.dtype) == (part.data_ptr(), *part.shape, E.BF) and m.stride == part.stride(0)
    column = t.float()[:, 3:4]  # of one column, whose distance to the next does not matter
    assert E.view(column).stride == 8 and E.view(column.t().contiguous().t()).cols == 1
    assert E.view(t[:0]).rows == 0


@pytest.mark.parametrize("make", [lambda t: t.t(), lambda t: t[:, ::2], lambda t: t.expand(2, 6, 8)[0].t(), lambda t: t[0],
                                  lambda t: t.half(), lambda t: t.double(), lambda t: t[:1].expand(6, 8)])
def test_what_would_be_read_wrongly_is_refused(make):
    """A transposed tensor, every other column, rows that are one and the same, other types than the library's."""
    import train_step as E
    with pytest.raises(ValueError):
        E.view(make(torch.zeros(6, 8, dtype=torch.bfloat16)))
