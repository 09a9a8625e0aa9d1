"""Page 0, which is read where keys have no page, holds infinities and NaN and is listed nowhere: no result changes."""
import math

import numpy as np
import pytest

from tests.paged_util import Batch, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("poison", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("new", [[1, 1, 1], [40, 70, 1], [1, 50, 200]], ids=str)
@pytest.mark.parametrize("page", [16, 64])
def test_page_zero_does_not_matter(page, new, poison):
    b = Batch([33, 100, 15], new, 4, 2, page=page, window=0, seed=61)
    # page 0 changes places with one that no table lists; then some entries are no page
    spare = sorted(set(range(b.n_pages)) - set(b.table[b.table < b.n_pages].tolist()))[0]
    for x in (b.k, b.v):
        x[spare] = x[0]
        x[0] = poison
    listed = b.table < 10 ** 6
    assert not (b.table[listed] == spare).any() or spare == 0
    b.table = np.where(listed & (b.table == 0), spare, b.table)
    b.table[1, 1] = -1
    b.table[2, 0] = b.n_pages
    b.run()
    check_attention(b)
