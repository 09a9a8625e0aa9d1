"""Attention over values at both ends of the number range: what a sum of weights of at most 1 holds, the kernels hold."""
import numpy as np
import pytest
import torch

from tests.paged_util import D, HALF_BF16, Batch, np64

pytestmark = pytest.mark.gpu


def rising(cached, new, heads, high, page=16):
    """Scores of 0, but for the keys `high`, which come late and weigh 2^7.5 more: less than makes the exponents' reference follow."""
    b = Batch(cached, new, *heads, page=page, seed=41)
    b.qkv[:b.rows] = 0
    b.qkv[:b.rows, :b.Hq * D:D] = 16                                # element 0 of every query head
    b.k[b.k == b.k] = 0
    for r, s in enumerate(b.seq):
        for j in high:
            if j < s:
                b.k[int(b.table[r, j // page]), :, j % page, 0] = 3.671875       # 16 * 3.671875 / sqrt(128) / ln 2 = 7.49
    return b


def check(b):
    """As in check_attention (the scores are exact up to their last rounding), without an absolute part."""
    o_ref, lse_ref, size = b.reference()
    o = np64(b.o[:b.rows, :b.Hq * D]).reshape(b.rows, b.Hq, D)
    assert np.isfinite(o).all(), f"{(~np.isfinite(o)).sum()} results are not finite"
    tol = 1.01 * (HALF_BF16 * np.abs(o_ref[:b.rows]) + (HALF_BF16 + 2.0 ** -12) * size[:b.rows])
    assert (np.abs(o - o_ref[:b.rows]) <= tol).all(), np.max(np.abs(o - o_ref[:b.rows]) / tol)
    assert (np.abs(np64(b.lse[:b.rows]) - lse_ref[:b.rows]) <= 2.0 ** -11).all()


CASES = {"few rows": ([700, 650, 700], [1, 1, 2], (128, 128)), "few rows, cut": ([5000], [1], (2, 1)), "tiles": ([630], [70], (4, 2)),
         "tiles, long": ([3000], [300], (8, 8))}


@pytest.mark.parametrize("scale", [1e37, 1e-34])
@pytest.mark.parametrize("case", list(CASES))
def test_large_and_small_values(case, scale):
    """Values of 1e37 times a weight of 2^7.5 leave fp32; at most eight such keys times 1 do not, and neither do thousands times 2^-7.5."""
    cached, new, heads = CASES[case]
    b = rising(cached, new, heads, [420, 421, 630, 1500, 2900])
    b.v.copy_((b.v.float().abs().clamp(0.5, 1) * scale).to(torch.bfloat16))
    b.run()
    check(b)
