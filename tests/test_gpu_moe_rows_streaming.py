"""Every variant of the row kernels, those that stream past the caches among them: matrices of more than 32, 128 and 256 MiB, against
plain indexing on the device in 64 bits.  That each case takes the variant it names is tested without a GPU (test_moe_train_choice.py)."""
import pytest
import torch

import paper_2503_20313_amd as tl
from tests.moe_train_util import BF16, HALF16, HALF32, I32, Lib

NAN = float("nan")
F64 = torch.float64

# variant, tokens, features, choices, rows of the sorted matrices.  Features: a row is a wave's and a workgroup's, the last piece of a row is not full.
FORWARD = [("dispatch cached cached", 2001, 776, 5, 9000), ("dispatch cached stream", 9001, 776, 5, 44000), ("dispatch cached stream", 3001, 2056, 5, 15005)]
SUMS = [(op + v, *s) for op in ("dispatch_grad", "combine") for v, *s in ((" cached cached", 9001, 776, 5, 44000), (" stream cached", 14001, 2056, 5, 70000),
                                                                          (" stream cached", 50001, 520, 6, 300006))]
GRADIENTS = [("combine_grad 1 cached cached", 2001, 776, 5, 9000), ("combine_grad 1 cached stream", 9001, 776, 5, 44000), ("combine_grad 1 stream stream", 20001, 776, 5, 100000),
             ("combine_grad 4 cached cached", 701, 2056, 5, 3400), ("combine_grad 4 cached stream", 3001, 2056, 5, 15005), ("combine_grad 4 stream stream", 7001, 2056, 5, 35000)]


class Inputs:
    def __init__(self, T, H, k, rows):
        self.T, self.H, self.k, self.rows = T, H, k, rows
        self.g = torch.Generator("cuda").manual_seed(T + H)
        # places in any order; every eighth choice is of another rank, places from `rows` on did not fit, the third token has no row
        pos = torch.randperm(T * k, device="cuda", generator=self.g).reshape(T, k)
        pos[torch.rand(T, k, device="cuda", generator=self.g) < 0.125] = -1
        pos[2] = -1
        self.part = (pos >= 0) & (pos < rows)
        self.pos, self.at = pos.to(I32), torch.where(self.part, pos, 0)
        self.w = torch.randn(T, k, device="cuda", generator=self.g)
        self.used = torch.where(self.part, self.w, 0.0)
        self.given = torch.where(self.part, self.w, NAN)          # the weight of a row that takes no part is not used
        self.named = torch.zeros(rows, dtype=torch.bool, device="cuda")
        self.named[pos[self.part]] = True

    def normal(self, n):
        return torch.randn(n, self.H, device="cuda", generator=self.g).to(BF16)

    def sorted_rows(self):
        m = self.normal(self.rows)
        m[~self.named] = NAN                                      # what no place names is not read
        return m

    def rows_of(self, m, j):
        """The rows of choice j in 64 bits, zeros where it takes no part."""
        return torch.where(self.part[:, j, None], m[self.at[:, j]].double(), 0.0)


def within(got, ref, bound, what):
    bad = ~((got.double() - ref).abs() <= bound)
    assert not bad.any().item(), f"{what}: {bad.sum().item()} of {bad.numel()} outside, first at {bad.nonzero()[0].tolist()}"


def name(v):
    return v.replace(" ", "_") if isinstance(v, str) else str(v)


@pytest.mark.gpu
@pytest.mark.parametrize("variant,T,H,k,rows", FORWARD, ids=name)
def test_dispatch(variant, T, H, k, rows):
    c = Inputs(T, H, k, rows)
    x = c.normal(T)
    xs, ref = (torch.full((rows + 1, H), 7.0, dtype=BF16, device="cuda") for _ in range(2))
    with Lib() as ctx:
        tl.tl_moe_dispatch(ctx, x, c.pos, T, H, k, rows, xs)
    for j in range(k):
        ref[c.at[c.part[:, j], j]] = x[c.part[:, j]]
    assert torch.equal(xs, ref)


@pytest.mark.gpu
@pytest.mark.parametrize("variant,T,H,k,rows", SUMS, ids=name)
def test_sums_of_a_tokens_rows(variant, T, H, k, rows):
    """A sum of n terms in fp32 is off by n half steps of the sum of their sizes, its bf16 by half a step of itself."""
    c = Inputs(T, H, k, rows)
    y, combine = c.sorted_rows(), variant.startswith("combine")
    add = c.normal(T) if combine else None
    out = torch.full((T + 1, H), 7.0, dtype=BF16, device="cuda")
    with Lib() as ctx:
        if combine:
            tl.tl_moe_combine(ctx, y, c.given, c.pos, T, H, k, rows, add, out)
        else:
            tl.tl_moe_dispatch_grad(ctx, y, c.pos, T, H, k, rows, out)
    ref = add.double() if combine else torch.zeros(T, H, dtype=F64, device="cuda")
    size = ref.abs()
    for j in range(k):
        row = c.rows_of(y, j) * (c.used[:, j, None].double() if combine else 1.0)
        ref += row
        size += row.abs()
    slack = (k + 1) * HALF32 * size
    within(out[:T], ref, HALF16 * (ref.abs() + slack) + slack, "out")
    assert (out[T] == 7).all().item()


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("variant,T,H,k,rows", GRADIENTS, ids=name)
def test_combine_grad(variant, T, H, k, rows, in_place):
    """dys: two roundings, to fp32 and to bf16; dtopk_w: a sum of H terms."""
    c = Inputs(T, H, k, rows)
    y, dout = c.sorted_rows(), c.normal(T)
    kept = y.clone()
    dys = y if in_place else torch.full((rows, H), 7.0, dtype=BF16, device="cuda")
    dw = torch.full((T, k), NAN, device="cuda")
    with Lib() as ctx:
        tl.tl_moe_combine_grad(ctx, dout, y, c.given, c.pos, T, H, k, rows, dys, dw)
    left = kept if in_place else torch.full((rows, H), 7.0, dtype=BF16, device="cuda")
    assert torch.equal(dys[~c.named].view(torch.int16), left[~c.named].view(torch.int16))
    for j in range(k):
        part, g = c.part[:, j], dout.double()
        ref = c.used[part, j, None].double() * g[part]
        within(dys[c.at[part, j]], ref, HALF16 * ref.abs() * (1 + 2.0 ** -15), "dys")
        terms = g * c.rows_of(kept, j)
        within(dw[:, j], terms.sum(1), H * HALF32 * terms.abs().sum(1), "dw")
        assert not dw[~part, j].any().item()


@pytest.mark.gpu
def test_lists_beyond_32_bits():
    """As many choices as there can be, row_pos and weights of more than 4 GiB each: the first, a middle and the last tokens have rows."""
    T, H, k, rows = (1 << 26) - 1, 8, 32, 64
    pos = torch.full((T, k), -1, dtype=I32, device="cuda")
    tokens = [0, 1 << 25, (1 << 26) - 3, T - 1]
    at = torch.randperm(rows, device="cuda", generator=torch.Generator("cuda").manual_seed(0))[:len(tokens) * 2].reshape(-1, 2)
    pos[tokens, 3], pos[tokens, k - 1] = at[:, 0].to(I32), at[:, 1].to(I32)
    x = torch.ones(T, H, dtype=BF16, device="cuda")
    x[tokens] = torch.arange(1, len(tokens) * H + 1, device="cuda").reshape(-1, H).to(BF16)
    xs, dx = torch.full((rows, H), 7.0, dtype=BF16, device="cuda"), torch.full_like(x, NAN)
    with Lib() as ctx:
        tl.tl_moe_dispatch(ctx, x, pos, T, H, k, rows, xs)
        ref = torch.full_like(xs, 7.0)
        ref[at[:, 0]], ref[at[:, 1]] = x[tokens], x[tokens]
        assert torch.equal(xs, ref)
        tl.tl_moe_dispatch_grad(ctx, xs, pos, T, H, k, rows, dx)
        has = torch.zeros(T, dtype=torch.bool, device="cuda")
        has[tokens] = True
        assert torch.equal(dx[tokens], 2 * x[tokens]) and not dx[~has].any().item()
        w = torch.full((T, k), NAN, device="cuda")
        w[tokens, 3], w[tokens, k - 1] = 2.0, 0.5
        tl.tl_moe_combine(ctx, xs, w, pos, T, H, k, rows, x, dx)
        assert torch.equal(dx[~has], x[~has]) and torch.equal(dx[tokens], (x[tokens] * 3.5).to(BF16))
        dw = torch.full((T, k), NAN, device="cuda")
        tl.tl_moe_combine_grad(ctx, x, xs, w, pos, T, H, k, rows, xs, dw)
        size = (x[tokens].float() ** 2).sum(1)
        assert torch.equal(xs[at[:, 0]], 2 * x[tokens]) and torch.equal(xs[at[:, 1]], 0.5 * x[tokens])
        assert torch.equal(dw[tokens, 3], size) and torch.equal(dw[tokens, k - 1], size)
        dw[tokens] = 0
        assert not dw.any().item()
