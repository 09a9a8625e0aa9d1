"""The slot maps' oracle counts what a request did not get without a limit of its own."""
import numpy as np
import pytest

from oracle import paged as ref


@pytest.mark.parametrize("new,T,max_new,over", [([300000], 1 << 13, 4096, 295904), ([300000], 1 << 18, 1 << 18, 37856), ([2 ** 31 - 1, 1], 16, 16, 2 ** 31 - 16),
                                                ([2 ** 31 - 1, 300], 16, 16, 2 ** 31 - 1), ([5, -3], 16, 16, 0)], ids=str)
def test_tokens_that_do_not_fit(new, T, max_new, over):
    w = ref.slots([0] * len(new), new, np.arange(20000), 0, np.zeros((len(new), 18750), np.int64), T, max_new, 16, 20000)
    assert w["counts"][3] == min(over, 2 ** 31 - 1)
