"""Every kernel that the experts' products can take, by name, on whole numbers: products and sums of small whole numbers are exact in fp32 in any order,
so that results equal those of plain fp32 products, rounded once.  That each case takes the kernel it names is tested without a GPU
(test_moe_train_choice.py)."""
import pytest
import torch

import paper_2503_20313_amd as tl
from tests.moe_train_util import BF16, F32, I32, Lib, product_ws

NAN = float("nan")
LEFT = 7.0                       # what rows hold that are no expert's
BEFORE, BEHIND = 1, 2            # rows that are no expert's

# rows of an expert: none, one, a row tile of the few-row kernel, one more, two, three, a whole unit, more than one, three and a bit
FEW = [0, 1, 16, 17, 33, 64, 65, 48] * 3 + [2, 0, 180, 32, 47, 3, 15, 5]
MIXED = [40] + [0] * 7 + [17] + [0] * 7
# kernel, rows of every expert, K, N.  Steps along the summed axis beyond what a ring holds, whole blocks of columns and a last one that is
# not, a last step that is short; tiles: whole, half and short ones of an expert, several rounds
PRODUCTS = [("gemm few wide 1 2", FEW, 2056, 1544), ("gemm few wide 2 1", [17, 40, 0, 64, 1, 33], 4104, 3592), ("gemm few narrow 2 1", [17, 40, 1, 33], 4104, 2824),
            ("gemm few narrow 4 1", MIXED, 2040, 136),
            ("gemm_grad_x few wide 1 2", FEW, 1544, 2056), ("gemm_grad_x few wide 2 1", [17, 40, 0, 64, 1, 33], 1800, 4104), ("gemm_grad_x few narrow 2 1", [17, 40, 1, 33], 1416, 4072),
            ("gemm_grad_x few narrow 4 1", MIXED, 72, 2040),
            ("gemm tiles 128 whole", [2000, 3, 0, 1100, 257, 20], 1032, 1800), ("gemm tiles 128 cut", [2000, 0, 60, 197], 4104, 2056),
            ("gemm tiles 256 whole", [5000, 0, 2300, 4700, 130, 3], 1032, 4104), ("gemm tiles 256 cut", [7000, 3, 400], 4104, 2056),
            ("gemm_grad_x tiles 128 whole", [2000, 3, 0, 1100, 257, 20], 1800, 1032), ("gemm_grad_x tiles 128 cut", [2000, 0, 60, 197], 2056, 4104),
            ("gemm_grad_x tiles 256 whole", [5000, 0, 2300, 4700, 130, 3], 4104, 1032), ("gemm_grad_x tiles 256 cut", [7000, 3, 400], 2056, 4104)]
GRADIENTS_OF_WEIGHTS = [("gemm_grad_w 128x128 whole", [700, 0, 1900], 264, 520), ("gemm_grad_w 128x128 cut", [4700, 0, 220], 264, 520),
                        ("gemm_grad_w 128x256 whole", [900, 150], 2056, 2056), ("gemm_grad_w 128x256 cut", [3000, 150], 2056, 2056),
                        ("gemm_grad_w 256x256 whole", [5000, 3, 0, 700, 2200, 1600, 900, 1500], 2056, 2056), ("gemm_grad_w 256x256 cut", [14300], 2056, 1032)]
# The buffer has room for more rows than there are: the kernel goes by the room.
ROOMY = [("gemm tiles 128 whole", FEW, 520, 264, 4000), ("gemm_grad_x tiles 128 whole", FEW, 264, 520, 4000), ("gemm_grad_w 128x128 cut", [64, 0, 17, 1], 264, 520, 9000)]


def room(counts):
    return BEFORE + sum(counts) + BEHIND


class Inputs:
    """Whole numbers in -2 .. 2; rows that are no expert's and the weights of experts without rows are NaN."""

    def __init__(self, counts, K, N, rows):
        g = torch.Generator("cuda").manual_seed(K + N + rows)
        ints = lambda *s: torch.randint(-2, 3, s, device="cuda", generator=g).to(BF16)
        self.counts, self.E, self.K, self.N, self.rows = counts, len(counts), K, N, rows
        self.at = [BEFORE]
        for n in counts:
            self.at.append(self.at[-1] + n)
        self.off = torch.tensor(self.at, dtype=I32, device="cuda")
        self.x, self.dy, self.w = ints(rows, K), ints(rows, N), ints(self.E, K, N)
        for m in (self.x, self.dy):
            m[:BEFORE] = NAN
            m[self.at[-1]:] = NAN
        for e, n in enumerate(counts):
            if n == 0:
                self.w[e] = NAN

    def spans(self):
        for e in range(self.E):
            if self.counts[e]:
                yield e, slice(self.at[e], self.at[e + 1])

    def product(self, ctx, name):
        """(the call's result, what it has to be)"""
        forward = name == "gemm"
        a, n = (self.x, self.N) if forward else (self.dy, self.K)
        out, ref = (torch.full((self.rows, n), LEFT, dtype=BF16, device="cuda") for _ in range(2))
        sizes = (self.rows, self.K, self.N, self.E)
        call, way = (tl.tl_moe_gemm, tl.TL_MOE_FORWARD) if forward else (tl.tl_moe_gemm_grad_x, tl.TL_MOE_GRAD_X)
        call(ctx, a, self.w, self.off, *sizes, out, *product_ws(ctx, way, *sizes))
        for e, rows in self.spans():
            w = self.w[e].float()
            ref[rows] = (a[rows].float() @ (w if forward else w.T.contiguous())).to(BF16)
        return out, ref

    def gradients_of_weights(self, ctx):
        sizes = (self.rows, self.K, self.N, self.E)
        ref = torch.zeros(self.E, self.K, self.N, device="cuda")
        for e, rows in self.spans():
            ref[e] = self.x[rows].float().T.contiguous() @ self.dy[rows].float()
        add = torch.randint(-9, 10, ref.shape, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).float()
        call = lambda dw, into=None: (tl.tl_moe_gemm_grad_w(ctx, self.x, self.dy, self.off, *sizes, into, dw, dw.dtype == F32,
                                                            *product_ws(ctx, tl.TL_MOE_GRAD_W, *sizes)), dw)[1]
        yield call(torch.full_like(ref, NAN, dtype=BF16)), ref.to(BF16)
        yield call(torch.full_like(ref, NAN)), ref
        yield call(torch.full_like(ref, NAN), add), ref + add
        total = ref + add
        yield call(add, add), total


def name(v):
    return v.replace(" ", "_") if isinstance(v, str) else f"E{len(v)}" if isinstance(v, list) else str(v)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,counts,K,N", PRODUCTS, ids=name)
def test_products(kernel, counts, K, N):
    c = Inputs(counts, K, N, room(counts))
    with Lib() as ctx:
        got, ref = c.product(ctx, kernel.split()[0])
        assert torch.equal(got, ref)
        assert torch.equal(c.product(ctx, kernel.split()[0])[0], got)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,counts,K,N", GRADIENTS_OF_WEIGHTS, ids=name)
def test_gradients_of_weights(kernel, counts, K, N):
    with Lib() as ctx:
        for got, ref in Inputs(counts, K, N, room(counts)).gradients_of_weights(ctx):
            assert torch.equal(got, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("kernel,counts,K,N,rows", ROOMY, ids=name)
def test_buffers_with_room_for_more_rows(kernel, counts, K, N, rows):
    c = Inputs(counts, K, N, rows)
    with Lib() as ctx:
        for got, ref in c.gradients_of_weights(ctx) if "grad_w" in kernel else [c.product(ctx, kernel.split()[0])]:
            assert torch.equal(got, ref)
