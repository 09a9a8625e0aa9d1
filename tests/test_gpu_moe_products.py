"""tl_moe_gemm, tl_moe_gemm_grad_x and tl_moe_gemm_grad_w against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from oracle import moe_train as o
from tests.moe_train_util import BF16, F32, I32, Lib, bf16_normal, gpu, host, product_ws, rounded, small_ints, within

pytestmark = pytest.mark.gpu
NAN = float("nan")
LEFT = 7.0              # what rows hold that are no expert's
FORWARD, GRAD_X, GRAD_W = tl.TL_MOE_FORWARD, tl.TL_MOE_GRAD_X, tl.TL_MOE_GRAD_W


class Call:
    """Inputs of all three products over `counts` rows, rows of no expert before and behind them; what no product may use is NaN."""

    def __init__(self, make, counts, K, N, before=0, behind=0):
        self.E, self.K, self.N = len(counts), K, N
        self.off = np.concatenate([[0], np.cumsum(counts)]) + before
        self.rows = self.off[-1] + behind
        (self.x, self.xr), (self.dy, self.dyr), (self.w, self.wr) = make(self.rows, K), make(self.rows, N), make(self.E, K, N)
        self.own = np.zeros(self.rows, bool)
        self.own[self.off[0]:self.off[-1]] = True
        for t in (self.x, self.dy):
            t[torch.from_numpy(~self.own).cuda()] = NAN
        for e, n in enumerate(counts):
            if n == 0:
                self.w[e] = NAN
        self.offd = gpu(self.off, I32)

    def sizes(self):
        return self.offd, int(self.rows), self.K, self.N, self.E

    def forward(self, ctx, ws=None):
        y = torch.full((self.rows, self.N), LEFT, dtype=BF16, device="cuda")
        tl.tl_moe_gemm(ctx, self.x, self.w, *self.sizes(), y, *(ws or product_ws(ctx, FORWARD, *self.sizes()[1:])))
        return y

    def grad_x(self, ctx, ws=None):
        dx = torch.full((self.rows, self.K), LEFT, dtype=BF16, device="cuda")
        tl.tl_moe_gemm_grad_x(ctx, self.dy, self.w, *self.sizes(), dx, *(ws or product_ws(ctx, GRAD_X, *self.sizes()[1:])))
        return dx

    def grad_w(self, ctx, dw, add=None, ws=None):
        tl.tl_moe_gemm_grad_w(ctx, self.x, self.dy, *self.sizes(), add, dw, dw.dtype == F32, *(ws or product_ws(ctx, GRAD_W, *self.sizes()[1:])))
        return dw

    def new_dw(self, dtype=BF16):
        return torch.full((self.E, self.K, self.N), NAN, dtype=dtype, device="cuda")


def to_bf16(a):
    return torch.from_numpy(a).to(F32).to(BF16).double().numpy()


# rows of every expert, K, N, rows of nobody in front and behind: single rows, empty experts, sums along fewer values than a step and than
# the ring of steps holds, tiles' edges and one beside them, more experts than compute units' worth of work
COUNTS = [([1], 8, 8, 0, 0), ([0], 16, 24, 0, 3), ([1, 0, 2], 72, 40, 0, 1), ([5, 0, 0, 64, 1], 136, 264, 2, 2), ([65, 63, 7], 256, 520, 0, 0),
          ([129, 127, 128], 512, 128, 0, 0), ([300, 0, 257], 264, 1032, 0, 5), ([256] * 3, 1000, 256, 1, 0), ([1] * 70, 64, 72, 0, 0), ([3, 1] * 128, 32, 16, 0, 0),
          ([700, 11], 40, 2056, 0, 0), ([1100], 776, 8, 0, 0), ([0, 0, 33], 2056, 96, 0, 0), ([2500, 3, 900, 0, 1], 264, 520, 0, 7),
          ([257, 2049, 255], 1288, 2072, 0, 0),
          # few tiles, long sums: cut
          ([1], 4104, 136, 0, 2), ([0, 130, 3], 2120, 264, 1, 0), ([70, 1], 264, 4168, 0, 0), ([200, 9], 136, 2120, 0, 3), ([3], 1000, 8200, 0, 0), ([100, 0, 59, 1], 2120, 2040, 0, 1),
          # few rows, a wide block of columns for two waves
          ([3, 0, 17, 40, 1, 2], 1992, 3208, 1, 0)]


def ints(seed):
    rng = np.random.default_rng(seed)
    return lambda *s: small_ints(rng, *s)


@pytest.mark.parametrize("counts,K,N,before,behind", COUNTS, ids=lambda v: str(v) if isinstance(v, int) else f"E{len(v)}x{max(v)}")
def test_whole_numbers_are_exact(counts, K, N, before, behind):
    """Products and sums of small whole numbers are exact in fp32 in any order: one rounding is left."""
    c = Call(ints(len(counts) + K), counts, K, N, before, behind)
    with Lib() as ctx:
        y, dx, dw, dw32 = c.forward(ctx), c.grad_x(ctx), c.grad_w(ctx, c.new_dw()), c.grad_w(ctx, c.new_dw(F32))
        add, add_ref = torch.full_like(dw32, 3.0), np.full(dw32.shape, 3.0)
        dw_add = c.grad_w(ctx, c.new_dw(F32), add)
        dw_own = c.grad_w(ctx, add, add)                   # in place
    for got, ref in ((y, o.products(c.xr, c.wr, c.off)), (dx, o.products_grad_x(c.dyr, c.wr, c.off))):
        assert np.array_equal(host(got)[c.own], to_bf16(ref[c.own])) and (host(got)[~c.own] == LEFT).all()
    ref = o.products_grad_w(c.xr, c.dyr, c.off)
    assert np.array_equal(host(dw), to_bf16(ref)) and np.array_equal(host(dw32), ref)
    assert np.array_equal(host(dw_add), ref + add_ref) and np.array_equal(host(dw_own), ref + add_ref)


def slack(n, size):
    """n products added in fp32 in any order, by an adder that may cut: a step a term."""
    return n * 2.0 ** -23 * size


# the large tiles (whole and with edges), a few rows of many experts against much of K, long sums into few tiles
@pytest.mark.parametrize("counts,K,N", [([700, 900, 300, 1000, 20, 0, 513, 400], 1032, 2120), ([2, 0, 1, 16, 17, 3] * 5, 2048, 776), ([3000, 1], 264, 136),
                                        ([40, 90], 4104, 72), ([5, 150, 0], 6152, 200), ([150, 30], 200, 6152)], ids=str)
def test_values(counts, K, N):
    rng = np.random.default_rng(K)
    c = Call(lambda *s: bf16_normal(rng, *s, scale=0.3), counts, K, N)
    with Lib() as ctx:
        y, dx, dw, dw32 = c.forward(ctx), c.grad_x(ctx), c.grad_w(ctx, c.new_dw()), c.grad_w(ctx, c.new_dw(F32))
        again = c.forward(ctx), c.grad_x(ctx), c.grad_w(ctx, c.new_dw()), c.grad_w(ctx, c.new_dw(F32))
    for a, b in zip((y, dx, dw, dw32), again):
        assert torch.equal(a, b)
    for got, ref, size, n in ((y, o.products(c.xr, c.wr, c.off), o.products(abs(c.xr), abs(c.wr), c.off), K),
                              (dx, o.products_grad_x(c.dyr, c.wr, c.off), o.products_grad_x(abs(c.dyr), abs(c.wr), c.off), N),
                              (dw, o.products_grad_w(c.xr, c.dyr, c.off), o.products_grad_w(abs(c.xr), abs(c.dyr), c.off), max(counts))):
        within(host(got), ref, rounded(ref, slack(n, size)))
    ref = o.products_grad_w(c.xr, c.dyr, c.off)
    within(host(dw32), ref, slack(max(counts), o.products_grad_w(abs(c.xr), abs(c.dyr), c.off)))


def test_gradients_against_differences():
    """<g, Y> is linear in X and in W: its difference along one row or one matrix is the gradient itself.  Whole numbers, exact."""
    c = Call(ints(77), [9, 0, 30], 64, 48)
    with Lib() as ctx:
        dx, dw = c.grad_x(ctx), c.grad_w(ctx, c.new_dw(F32))
        base = host(c.forward(ctx))
        for row, e in ((0, 0), (8, 0), (9, 2), (38, 2)):
            for k in (0, 13, 63):
                c.x[row, k] += 1
                diff = host(c.forward(ctx)) - base
                c.x[row, k] -= 1
                assert (diff[row] * c.dyr[row]).sum() == o.products_grad_x(c.dyr, c.wr, c.off)[row, k] and not np.delete(diff, row, 0).any()
                n = (k * 7) % 48
                c.w[e, k, n] += 1
                diff = host(c.forward(ctx)) - base
                c.w[e, k, n] -= 1
                assert (diff * c.dyr).sum() == host(dw)[e, k, n]
    assert np.array_equal(host(dx), to_bf16(o.products_grad_x(c.dyr, c.wr, c.off)))


@pytest.mark.parametrize("K,N", [(64, 72), (2120, 72)])      # a sum in one piece, and cut
def test_offsets_that_leave_the_rows_are_cut(K, N):
    """Rows from max_rows on are not there, whatever expert_offsets says; the rest is as it would be."""
    c = Call(ints(5), [100, 50, 60], K, N)
    c.offd = gpu([0, 100, 150, 1 << 30], I32)
    with Lib() as ctx:
        y, dw = c.forward(ctx), c.grad_w(ctx, c.new_dw())
        assert np.array_equal(host(y), to_bf16(o.products(c.xr, c.wr, c.off))) and np.array_equal(host(dw), to_bf16(o.products_grad_w(c.xr, c.dyr, c.off)))
        c.offd = gpu([-5, 100, 90, 1 << 30], I32)           # an expert that ends before it starts has no rows
        off = np.array([0, 100])
        y = host(c.forward(ctx))
        assert np.array_equal(y[:90], to_bf16(o.products(c.xr[:100], c.wr[:1], off))[:90])
        assert not host(c.grad_w(ctx, c.new_dw()))[1].any()


# a round and a few tiles, small and large, of which some are whole, half, and at an edge; no whole round; a round of small ones and a bit
@pytest.mark.parametrize("counts,K,N", [([2000, 0, 60, 197], 4104, 2056), ([7000, 3, 400], 4104, 2056), ([3, 300, 120], 6152, 264), ([4100, 70], 4104, 1032)], ids=str)
def test_last_round_is_cut(counts, K, N):
    """Whole numbers, against products in fp32, which are exact; dX of the matrices the other way round."""
    with Lib() as ctx:
        for way, c in ((FORWARD, Call(ints(K), counts, K, N, 1, 2)), (GRAD_X, Call(ints(N), counts, N, K, 1, 2))):
            assert tl.tl_moe_gemm_query(ctx, way, *c.sizes()[1:]) > 256          # (room for parts)
            got, again = [c.forward(ctx) if way == FORWARD else c.grad_x(ctx) for _ in range(2)]
            ref = torch.full_like(got, LEFT)
            for e in range(c.E):
                lo, hi = int(c.off[e]), int(c.off[e + 1])
                w = c.w[e].float()
                ref[lo:hi] = (c.x[lo:hi].float() @ w if way == FORWARD else c.dy[lo:hi].float() @ w.T.contiguous()).to(BF16)
            assert torch.equal(got, ref) and torch.equal(got, again)


# tiles of the three shapes, their sums cut and not
@pytest.mark.parametrize("counts,K,N,cut", [([4700, 0, 220], 264, 520, True), ([3000, 150], 2056, 2056, True), ([14300], 2056, 1032, True), ([700, 0, 1900], 264, 520, False),
                                            ([900, 150], 2056, 2056, False), ([5000, 3, 0, 700, 2200, 1600, 900, 1500], 2056, 2056, False)], ids=str)
def test_gradients_of_weights_over_long_sums(counts, K, N, cut):
    """Whole numbers, against products in fp32, which are exact."""
    c = Call(ints(K + N), counts, K, N, 1, 2)
    ref = torch.zeros(c.E, K, N, device="cuda")
    for e in range(c.E):
        rows = slice(int(c.off[e]), int(c.off[e + 1]))
        if counts[e]:
            ref[e] = c.x[rows].float().T.contiguous() @ c.dy[rows].float()
    add = torch.arange(K * N, device="cuda").remainder(17).float().reshape(K, N).expand(c.E, K, N).contiguous()
    with Lib() as ctx:
        assert (tl.tl_moe_gemm_query(ctx, GRAD_W, *c.sizes()[1:]) > 1 << 20) == cut
        for _ in range(2):
            assert torch.equal(c.grad_w(ctx, c.new_dw()), ref.to(BF16)) and torch.equal(c.grad_w(ctx, c.new_dw(F32)), ref)
            assert torch.equal(c.grad_w(ctx, c.new_dw(F32), add), ref + add)
        total = ref + add
        assert torch.equal(c.grad_w(ctx, add, add), total)


def test_experts_whose_rows_overlap_stay_inside_workspace_and_results():
    """More tiles than there can be: nothing is written beside workspace and results."""
    c = Call(ints(6), [300], 4104, 136)
    E, n = 16, tl.tl_moe_gemm_query
    w = torch.zeros(E, 4104, 136, dtype=BF16, device="cuda")
    off = gpu([0, 300] * 8 + [0], I32)
    with Lib() as ctx:
        need = n(ctx, FORWARD, 300, 4104, 136, E)
        assert need > 256                                   # (a cut sum)
        ws = torch.full((need // 4 + 1024,), -1, dtype=I32, device="cuda")
        y = torch.full((301, 136), LEFT, dtype=BF16, device="cuda")
        tl.tl_moe_gemm(ctx, c.x, w, off, 300, 4104, 136, E, y, ws, need)
        torch.cuda.synchronize()
        assert (ws[need // 4:] == -1).all() and (host(y)[300] == LEFT).all()


def test_one_workspace_for_all():
    """Calls of different kinds and sizes that follow each other, on one workspace that is large enough for each."""
    with Lib() as ctx:
        calls = [Call(ints(i), counts, K, N) for i, (counts, K, N) in enumerate([([2000], 256, 136), ([1, 1, 3], 4096, 64), ([300] * 4, 128, 512)])]
        n = max(tl.tl_moe_gemm_query(ctx, way, *c.sizes()[1:]) for c in calls for way in (FORWARD, GRAD_X, GRAD_W))
        ws = (torch.full((n // 4,), -1, dtype=I32, device="cuda"), n)
        for _ in range(2):
            for c in calls:
                y, dw, dx = c.forward(ctx, ws), c.grad_w(ctx, c.new_dw(), ws=ws), c.grad_x(ctx, ws)
                assert np.array_equal(host(y), to_bf16(o.products(c.xr, c.wr, c.off)))
                assert np.array_equal(host(dx), to_bf16(o.products_grad_x(c.dyr, c.wr, c.off)))
                assert np.array_equal(host(dw), to_bf16(o.products_grad_w(c.xr, c.dyr, c.off)))


def test_values_that_are_not_finite_stay_with_their_expert():
    c = Call(ints(12), [40, 30, 50], 128, 136)
    c.x[45, 3], c.dy[45, 7] = float("inf"), NAN
    with Lib() as ctx:
        y, dx, dw = host(c.forward(ctx)), host(c.grad_x(ctx)), host(c.grad_w(ctx, c.new_dw()))
    assert np.isfinite(np.delete(y, 45, 0)).all() and np.isfinite(np.delete(dx, 45, 0)).all() and np.isnan(dx[45]).all()
    assert np.isfinite(dw[[0, 2]]).all() and np.isnan(dw[1, :, 7]).all() and not np.isfinite(dw[1, 3]).all()
    rest = np.delete(np.delete(dw[1], 3, 0), 7, 1)
    assert np.isfinite(rest).all()


def test_rows_and_weights_beyond_32_bits():
    """Matrices of more than 2^31 elements: the last expert, the last rows."""
    K, N, E = 8192, 2048, 140                               # 2.3e9 weights
    w = torch.zeros(E, K, N, dtype=BF16, device="cuda")
    rng = np.random.default_rng(3)
    wl, wlr = small_ints(rng, K, N)
    w[E - 1] = wl
    rows = (1 << 31) // K + 40
    x = torch.zeros(rows, K, dtype=BF16, device="cuda")
    xl, xlr = small_ints(rng, 30, K)
    x[rows - 30:] = xl
    off = gpu([0] * E + [rows], I32)
    off[E - 1] = rows - 30
    dyl, dylr = small_ints(rng, 30, N)
    with Lib() as ctx:
        y = torch.zeros(rows, N, dtype=BF16, device="cuda")
        tl.tl_moe_gemm(ctx, x, w, off, rows, K, N, E, y, *product_ws(ctx, FORWARD, rows, K, N, E))
        torch.cuda.synchronize()
        assert np.array_equal(host(y[rows - 30:]), to_bf16(xlr @ wlr))
        y[rows - 30:] = dyl
        dw = torch.full((E, K, N), NAN, dtype=BF16, device="cuda")
        tl.tl_moe_gemm_grad_w(ctx, x, y, off, rows, K, N, E, None, dw, False, *product_ws(ctx, GRAD_W, rows, K, N, E))
        torch.cuda.synchronize()
        assert np.array_equal(host(dw[E - 1]), to_bf16(xlr.T @ dylr)) and not dw[0].any() and not dw[E - 2].any()
        tl.tl_moe_gemm_grad_x(ctx, y, w, off, rows, K, N, E, x, *product_ws(ctx, GRAD_X, rows, K, N, E))
        torch.cuda.synchronize()
        assert np.array_equal(host(x[rows - 30:]), to_bf16(dylr @ wlr.T))
