"""tl_moe_sort against its definition: whole numbers, equal."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from oracle import moe_train as o
from tests.moe_train_util import I32, Lib, choose, gpu, sort_call

pytestmark = pytest.mark.gpu


def check(ids, first, E, got):
    off, order, pos = o.sort_rows(ids, first, E)
    n = len(order)
    assert np.array_equal(got[0].cpu().numpy(), off)
    assert np.array_equal(got[1].cpu().numpy()[:n], order) and (got[1].cpu().numpy()[n:] == -7).all()
    assert np.array_equal(got[2].cpu().numpy(), pos)


# one chunk of rows and several, up to each count of rows a thread, at the borders of waves and chunks
@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 2, 8), (5, 3, 4), (64, 1, 2), (63, 8, 64), (128, 8, 256), (1025, 1, 5), (341, 3, 7), (342, 3, 7), (2048, 2, 33),
                                   (4097, 5, 60), (16381, 8, 64), (16384, 8, 256), (16385, 8, 129), (40000, 7, 16), (131072, 8, 256)])
@pytest.mark.parametrize("ranks", [1, 3])
def test_sort(T, k, E, ranks):
    rng = np.random.default_rng(T * 31 + k + E)
    k = min(k, E * ranks)
    ids = choose(rng, T, E * ranks, k) if E * ranks * T < 1 << 24 else rng.integers(0, E * ranks, size=(T, k))
    with Lib() as ctx:
        first = E * (ranks // 2)
        check(ids, first, E, sort_call(ctx, gpu(ids, I32), first, E))


def test_any_id_is_safe_and_none_of_ours_takes_no_part():
    rng = np.random.default_rng(5)
    ids = rng.integers(-3, 12, size=(700, 4))
    ids[::9] = [-(1 << 31), (1 << 31) - 1, -1, 8]
    with Lib() as ctx:
        check(ids, 0, 8, sort_call(ctx, gpu(ids, I32), 0, 8))
        check(ids, 4, 3, sort_call(ctx, gpu(ids, I32), 4, 3))
        none = np.full((33, 2), -1)
        check(none, 0, 8, sort_call(ctx, gpu(none, I32), 0, 8))
        one = np.full((3000, 4), 6)                     # all rows of one expert, the same one several times in a token
        check(one, 0, 8, sort_call(ctx, gpu(one, I32), 0, 8))
        far = np.full((40, 1), (1 << 31) - 1)           # the last expert there can be
        check(far, (1 << 31) - 256, 256, sort_call(ctx, gpu(far, I32), (1 << 31) - 256, 256))


def test_the_order_is_that_of_the_router():
    T, E, k = 3000, 32, 5
    with Lib() as ctx:
        logits = torch.randn(T, E, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
        ids, rows = torch.zeros(T, k, dtype=I32, device="cuda"), torch.zeros(T * k, dtype=I32, device="cuda")
        w, off, nt = torch.zeros(T, k, device="cuda"), torch.zeros(E + 1, dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda")
        tab = torch.zeros(-(-T * k // 128) + E, 8, dtype=I32, device="cuda")
        tl.tl_moe_route(ctx, logits, T, E, k, 1, 128, ids, w, off, rows, tab, nt)
        got = sort_call(ctx, ids, 0, E)
        torch.cuda.synchronize()
        assert torch.equal(got[0], off) and torch.equal(got[1], rows)


def test_calls_share_a_workspace():
    """Two sizes in turn, and twice the same, on one workspace and another stream."""
    rng = np.random.default_rng(8)
    with Lib() as ctx:
        ws = torch.full((1 << 16,), 12345, dtype=I32, device="cuda")
        s = torch.cuda.Stream()
        torch.cuda.synchronize()
        for T, k, E in [(9000, 3, 60), (2000, 8, 256), (9000, 3, 60), (1, 1, 3)]:
            ids = choose(rng, T, E, k)
            g = gpu(ids, I32)
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                got = sort_call(ctx, g, 0, E, s, ws)
            s.synchronize()
            check(ids, 0, E, got)
