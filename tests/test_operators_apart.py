"""Which arrays the training operators take to overlap: against sets of bytes (CPU, addresses are never read).

Every call here ends at its check of the arrays: a pair that is apart is followed by one that overlaps for certain."""
import random

import pytest

from paper_2609_27193_amd import layercheck as LC

B, F = LC.LC_DT_BF16, LC.LC_DT_F32
BASE = 0x7F0000000000
FAR = BASE + (1 << 36)
NORM = LC.norm_params(LC.LC_NORM_LAYER, 0, 0, F, 1e-5)


def said(call):
    with pytest.raises(LC.LCError) as e:
        call()
    assert e.value.code == LC.LC_ERR_INVALID_ARG
    return str(e.value)


def bytes_of(at, rows, width, pitch):
    return {at + r * pitch + i for r in range(rows) for i in range(width)}


def test_a_vector_or_a_row_between_the_rows_of_another_array():
    """The statistics of a norm beside the columns of its result, and one token's row beside the rows of a table."""
    y = LC.matrix(BASE, 4, 8, B, 32)      # 16 bytes of every 64
    x = LC.matrix(FAR, 4, 8, B)
    beside = dict(mean=BASE + 16, rstd=BASE + 16)  # apart from y; that they are one array is what is wrong
    assert "mean and rstd" in said(lambda: LC.lc_norm_forward(NORM, x, y, **beside))
    assert "y and mean" in said(lambda: LC.lc_norm_forward(NORM, x, y, mean=BASE + 12))
    assert "y and mean" in said(lambda: LC.lc_norm_forward(NORM, x, y, mean=BASE + 64 + 48 + 4))
    out = LC.matrix(BASE + 16, 1, 8, B)
    weight = LC.matrix(BASE, 4, 8, B, 32)
    assert "out and tokens" in said(lambda: LC.lc_embedding_forward(weight, BASE + 24, LC.LC_IT_I64, 1, out))
    assert "out and weight" in said(lambda: LC.lc_embedding_forward(weight, FAR, LC.LC_IT_I64, 1, LC.matrix(BASE + 64 - 8, 1, 8, B)))


def test_pairs_of_arrays_against_their_bytes():
    """lc_norm_forward's y against its mean and against its x; what is apart goes on to rstd, which is y itself."""
    rng = random.Random(1)
    for _ in range(4000):
        rows, cols = rng.choice([1, 2, 3, 5]), rng.randrange(1, 9)
        stride = cols + rng.randrange(0, 12)
        y = LC.matrix(BASE, rows, cols, F, stride)
        mine = bytes_of(BASE, rows, 4 * cols, 4 * stride)
        at = BASE + 4 * rng.randrange(-24, 80)
        if rng.random() < 0.5:  # a vector of rows floats
            text = said(lambda: LC.lc_norm_forward(NORM, LC.matrix(FAR, rows, cols, F), y, mean=at, rstd=BASE))
            apart = not mine & bytes_of(at, 1, 4 * rows, 0)
            assert ("y and mean" not in text) == apart, (rows, cols, stride, at - BASE)
        else:  # x in rows of the same pitch; of one row, wherever it lies
            text = said(lambda: LC.lc_norm_forward(NORM, LC.matrix(at, rows, cols, F, stride), y, mean=FAR, rstd=FAR))
            apart = not mine & bytes_of(at, rows, 4 * cols, 4 * stride)
            assert ("y and x" not in text) == apart, (rows, cols, stride, at - BASE)
