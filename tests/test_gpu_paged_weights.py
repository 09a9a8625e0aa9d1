"""Few rows (at most 32 per key head): the weights enter the product with V with more bits than bf16 has."""
import numpy as np
import pytest

from tests.paged_util import D, HALF_BF16, Batch, check_attention, np64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,cached,new", [((2, 1), [1, 2, 5, 31, 200], [1] * 5), ((16, 2), [700, 1, 40], [1, 1, 1]), ((32, 1), [64, 3], [1, 1]), ((5, 1), [90, 2], [6, 1]),
                                              ((4, 1), [6000], [1]), ((4, 2), [100, 1, 2, 3], [90, 1, 1, 1])], ids=str)
@pytest.mark.parametrize("window", [0, 50])
def test_error_of_the_results(heads, cached, new, window):
    """A result's own rounding is half a step.  A weight is kept as two bf16 numbers, its first 8 bits and then the rest, under 2^-7 of it, to half a
    step: off by 2^-15 at most.  The fp32 scores move weights by under 2^-12 (as in check_attention).  With weights of one bf16 number it
    would be 2^-8."""
    b = Batch(cached, new, *heads, page=16, window=window, seed=51)
    b.run()
    few = np.concatenate([np.full(n, n * heads[0] // heads[1] <= 32) for n in new])
    o_ref, _, size = (x[:b.rows] for x in b.reference())
    o = np64(b.o[:b.rows, :b.Hq * D]).reshape(b.rows, b.Hq, D)
    tol = 1.01 * (HALF_BF16 * np.abs(o_ref) + (2.0 ** -15 + 2.0 ** -12) * size) + 1e-30
    assert (np.abs(o - o_ref) <= tol)[few].all(), np.max((np.abs(o - o_ref) / tol)[few])


@pytest.mark.parametrize("kind", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("heads", [(2, 1), (16, 1)], ids=str)
def test_values_that_every_row_sees(kind, heads):
    """Infinities in keys that all rows of a request see, under weights of all sizes: the second part of a weight adds no NaN."""
    b = Batch([300, 2000], [2, 1], *heads, page=16, seed=52)
    for r, at in ((0, 0), (0, 77), (1, 5), (1, 64), (1, 1990)):
        b.v[int(b.table[r, at // 16]), :, at % 16, 3 + at % 100] = kind
    b.qkv[:b.rows, :b.Hq * D] = 0                     # equal scores: every weight is a power of two, whose second part would be zero
    b.run()
    check_attention(b)
