"""tl_moe_dispatch, tl_moe_combine and their gradients against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from oracle import moe_train as o
from tests.moe_train_util import BF16, F32, HALF16, HALF32, I32, Lib, bf16_normal, gpu, host, places, rounded, within

pytestmark = pytest.mark.gpu
NAN = float("nan")

# T, H, topk, experts, ranks, room: one token, rows shorter than a wave's piece and longer than a workgroup's, odd numbers of pieces,
# ranks that hold a part of the experts, full buffers
CASES = [(1, 8, 1, 2, 1, 1), (1, 4096, 2, 8, 1, 1), (3, 520, 3, 4, 1, 1), (17, 1032, 5, 8, 4, 1), (64, 2056, 2, 8, 2, 0.7), (33, 4104, 8, 16, 1, 0.5),
         (5, 8192, 32, 64, 1, 1), (2, 20488, 4, 8, 1, 1), (300, 136, 6, 8, 3, 1), (1000, 64, 2, 4, 1, 0.9), (7, 512, 4, 4, 9, 1),
         (9, 1024, 7, 16, 1, 0.8), (50, 776, 32, 64, 2, 1)]


def setup(T, H, k, E, ranks, room):
    rng = np.random.default_rng(T + H * 3 + k * 7)
    pos = places(rng, T, k, E, ranks)[2]
    rows = max(1, int(T * k * room))
    part = (pos >= 0) & (pos < rows)
    return rng, pos, rows, part


@pytest.mark.parametrize("T,H,k,E,ranks,room", CASES)
def test_dispatch(T, H, k, E, ranks, room):
    rng, pos, rows, part = setup(T, H, k, E, ranks, room)
    x, xr = bf16_normal(rng, T, H)
    xs = torch.full((rows + 1, H), 7.0, dtype=BF16, device="cuda")
    with Lib() as ctx:
        tl.tl_moe_dispatch(ctx, x, gpu(pos, I32), T, H, k, rows, xs)
    ref = o.dispatch(xr, pos, np.full((rows, H), 7.0))
    assert np.array_equal(host(xs)[:rows], ref)          # rows that nobody's place names stay as they were
    assert (host(xs)[rows] == 7).all()


@pytest.mark.parametrize("T,H,k,E,ranks,room", CASES)
def test_dispatch_grad(T, H, k, E, ranks, room):
    rng, pos, rows, part = setup(T, H, k, E, ranks, room)
    d, dr = bf16_normal(rng, rows, H)
    taken = np.zeros(rows, bool)
    taken[pos[part]] = True
    d[torch.from_numpy(~taken).cuda()] = NAN              # what no token names is not read
    dx = torch.full((T + 1, H), 7.0, dtype=BF16, device="cuda")
    with Lib() as ctx:
        tl.tl_moe_dispatch_grad(ctx, d, gpu(pos, I32), T, H, k, rows, dx)
    ref = o.dispatch_grad(dr, pos)
    within(host(dx)[:T], ref, rounded(ref, k * HALF32 * o.dispatch_grad(np.abs(dr), pos)), "dx")
    assert (host(dx)[T] == 7).all()


@pytest.mark.parametrize("add", [False, True, "in place"])
@pytest.mark.parametrize("T,H,k,E,ranks,room", CASES)
def test_combine(T, H, k, E, ranks, room, add):
    rng, pos, rows, part = setup(T, H, k, E, ranks, room)
    y, yr = bf16_normal(rng, rows, H)
    a, ar = bf16_normal(rng, T, H, scale=2.0)
    w = rng.normal(size=(T, k)).astype(np.float32)
    wd = w.copy()
    wd[~part] = NAN                                        # the weight of a row that takes no part is not used
    out = a if add == "in place" else torch.full((T, H), NAN, dtype=BF16, device="cuda")
    with Lib() as ctx:
        tl.tl_moe_combine(ctx, y, gpu(wd, F32), gpu(pos, I32), T, H, k, rows, a if add else None, out)
    ref = o.combine(yr, w.astype(np.float64), pos, ar if add else None)
    size = o.combine(np.abs(yr), np.abs(w).astype(np.float64), pos, np.abs(ar) if add else None)
    within(host(out), ref, rounded(ref, (k + 1) * HALF32 * size), "out")


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("T,H,k,E,ranks,room", CASES)
def test_combine_grad(T, H, k, E, ranks, room, in_place):
    rng, pos, rows, part = setup(T, H, k, E, ranks, room)
    y, yr = bf16_normal(rng, rows, H)
    g, gr = bf16_normal(rng, T, H, scale=0.1)
    w = rng.normal(size=(T, k)).astype(np.float32)
    wd = w.copy()
    wd[~part] = NAN
    dys = y if in_place else torch.full((rows, H), 7.0, dtype=BF16, device="cuda")
    dw = torch.full((T, k), NAN, dtype=F32, device="cuda")
    with Lib() as ctx:
        tl.tl_moe_combine_grad(ctx, g, y, gpu(wd, F32), gpu(pos, I32), T, H, k, rows, dys, dw)
    dys_ref, dw_ref = o.combine_grad(gr, yr, w.astype(np.float64), pos, yr if in_place else np.full((rows, H), 7.0))
    within(host(dys), dys_ref, HALF16 * np.abs(dys_ref) * (1 + 2.0 ** -15), "dys")     # two roundings: 2^-8 + 2^-24 and their product
    size = o.combine_grad(np.abs(gr), np.abs(yr), np.abs(w), pos, np.zeros((rows, H)))[1]
    within(host(dw), dw_ref, H * HALF32 * size, "dw")
    assert (host(dw)[~part] == 0).all()


def test_a_token_without_rows():
    T, H, k, rows = 6, 72, 3, 10
    pos = np.array([[-1, -1, -1], [4, -1, 10], [-(1 << 31), (1 << 31) - 1, 11], [0, 1, 2], [-1, 9, -1], [10, 10, 10]])
    rng = np.random.default_rng(1)
    (y, yr), (a, ar) = bf16_normal(rng, rows, H), bf16_normal(rng, T, H)
    ones, p = torch.ones(T, k, device="cuda"), gpu(pos, I32)
    out, plain, dx = (torch.full((T, H), NAN, dtype=BF16, device="cuda") for _ in range(3))
    dw = torch.full((T, k), NAN, device="cuda")
    with Lib() as ctx:
        tl.tl_moe_combine(ctx, y, ones, p, T, H, k, rows, a, out)
        tl.tl_moe_combine(ctx, y, ones, p, T, H, k, rows, None, plain)
        tl.tl_moe_dispatch_grad(ctx, y, p, T, H, k, rows, dx)
        tl.tl_moe_combine_grad(ctx, a, y, ones, p, T, H, k, rows, y, dw)
    for t in (0, 2, 5):
        assert np.array_equal(host(out)[t], ar[t]) and not host(plain)[t].any() and not host(dx)[t].any() and not host(dw)[t].any()
    assert np.array_equal(host(y)[[3, 5, 6, 7, 8]], yr[[3, 5, 6, 7, 8]])      # rows that no place names


def test_values_that_are_not_finite_stay_with_their_token():
    T, H, k = 40, 264, 2
    rng, pos, rows, part = setup(T, H, k, 4, 1, 1)
    y, yr = bf16_normal(rng, rows, H)
    g, gr = bf16_normal(rng, T, H)
    y[pos[7, 0], 5], y[pos[9, 1], 3], g[11, 0] = float("inf"), NAN, float("-inf")
    w = torch.ones(T, k, device="cuda")
    w[13, 0] = 0.0
    y[pos[13, 0], 2] = float("inf")
    out, dw, dys = torch.zeros(T, H, dtype=BF16, device="cuda"), torch.zeros(T, k, device="cuda"), torch.zeros(rows, H, dtype=BF16, device="cuda")
    with Lib() as ctx:
        tl.tl_moe_combine(ctx, y, w, gpu(pos, I32), T, H, k, rows, None, out)
        tl.tl_moe_combine_grad(ctx, g, y, w, gpu(pos, I32), T, H, k, rows, dys, dw)
    bad = np.argwhere(~np.isfinite(host(out)))
    assert bad.tolist() == [[7, 5], [9, 3], [13, 2]] and host(out)[7, 5] == np.inf and np.isnan(host(out)[13, 2])    # 0 * inf, as the formula has it
    assert np.argwhere(~np.isfinite(host(dys))).tolist() == sorted([pos[11, j], 0] for j in range(k))
    assert sorted(map(tuple, np.argwhere(~np.isfinite(host(dw))))) == sorted([(7, 0), (9, 1), (11, 0), (11, 1), (13, 0)])


def test_matrices_beyond_32_bits():
    """Sorted rows of more than 4 GiB, and of more than 2^31 elements: the first and the last rows."""
    T, H, k = 4, 8192, 1
    rows = (1 << 31) // H + 3
    pos = np.array([[0], [rows - 1], [rows // 2 + 1], [-1]])
    rng = np.random.default_rng(2)
    x, xr = bf16_normal(rng, T, H)
    xs = torch.zeros(rows, H, dtype=BF16, device="cuda")
    p, out, w, dw = gpu(pos, I32), torch.zeros(T, H, dtype=BF16, device="cuda"), torch.ones(T, k, device="cuda"), torch.zeros(T, k, device="cuda")
    with Lib() as ctx:
        tl.tl_moe_dispatch(ctx, x, p, T, H, k, rows, xs)
        torch.cuda.synchronize()
        for t in range(3):
            assert np.array_equal(host(xs[pos[t, 0]]), xr[t])
        tl.tl_moe_combine(ctx, xs, w, p, T, H, k, rows, None, out)
        torch.cuda.synchronize()
        assert np.array_equal(host(out)[:3], xr[:3]) and not host(out)[3].any()
        tl.tl_moe_combine_grad(ctx, x, xs, w, p, T, H, k, rows, xs, dw)
        torch.cuda.synchronize()
        ref = (xr[:3] ** 2).sum(1)
        within(host(dw)[:3, 0], ref, H * HALF32 * ref, "dw")
