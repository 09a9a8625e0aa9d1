"""tl_moe_route_grad against its definition in 64 bits, and against differences of tl_moe_route's own weights."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from oracle import moe_train as o
from tests.moe_train_util import F32, I32, Lib, choose, gpu, host, within

pytestmark = pytest.mark.gpu


def grad(logits, ids, dw, renormalize, in_place=False):
    T, E = logits.shape
    l = gpu(logits, F32)
    d = l if in_place else torch.full((T, E), float("nan"), device="cuda")
    with Lib() as ctx:
        tl.tl_moe_route_grad(ctx, l, gpu(ids, I32), gpu(dw, F32), T, E, ids.shape[1], renormalize, d)
    return host(d)


def bound(logits, ids, dw, renormalize):
    """An exponential is off by 2 steps and by what the rounding of its argument |l - top| does, a sum of n terms by n half steps, and
    every result is a sum of at most topk products of such numbers with dw: c half steps of the sum of their sizes."""
    T, E = logits.shape
    k = ids.shape[1]
    real = (ids >= 0) & (ids < E)
    w = o.route_weights(logits, ids, renormalize)
    share = w if renormalize else None
    mean = (np.abs(dw) * w).sum(1, keepdims=True)
    size = np.zeros((T, E))
    for t, j in zip(*np.nonzero(real)):
        size[t, ids[t, j]] += w[t, j] * (abs(dw[t, j]) + (mean[t, 0] if renormalize else 0))
    if not renormalize:
        with np.errstate(invalid="ignore"):
            p = np.exp(logits - logits.max(1, keepdims=True))
            size += np.nan_to_num(p / p.sum(1, keepdims=True)) * mean
    finite = np.where(np.isfinite(logits), logits, 0)
    c = 2 * (E + 2 * k + 16) + np.abs(finite - finite.max(1, keepdims=True)).max(1, keepdims=True)
    return c * 2.0 ** -24 * size + 1e-37


@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 2, 2), (5, 5, 3), (33, 8, 8), (100, 9, 2), (257, 16, 4), (64, 31, 5), (1000, 32, 32), (77, 60, 6), (4097, 64, 8), (50, 65, 7),
                                   (129, 128, 32), (3, 129, 1), (700, 256, 8)])
def test_gradient(T, E, k, renormalize):
    rng = np.random.default_rng(T + E * 5 + k)
    logits = (rng.normal(size=(T, E)) * 3).astype(np.float32).astype(np.float64)
    ids = np.argsort(-logits, axis=1, kind="stable")[:, :k] if T % 2 else choose(rng, T, E, k)
    dw = rng.normal(size=(T, k)).astype(np.float32).astype(np.float64)
    ref = o.route_grad(logits, ids, dw, renormalize)
    within(grad(logits, ids, dw, renormalize, in_place=T > 500), ref, bound(logits, ids, dw, renormalize), "dlogits")


@pytest.mark.parametrize("renormalize", [False, True])
def test_masked_experts_and_choices_that_are_none(renormalize):
    rng = np.random.default_rng(9)
    T, E, k = 12, 40, 4
    logits = rng.normal(size=(T, E)).astype(np.float32).astype(np.float64)
    ids = choose(rng, T, E, k)
    logits[0] = -np.inf                      # nothing left
    logits[1, :39] = -np.inf                 # one left, chosen
    ids[1] = [39, 0, 1, 2]
    logits[2, ::2] = -np.inf                 # masked ones among the chosen
    ids[2] = [0, 2, 4, 5]
    ids[3] = -1                              # a dropped token
    ids[4, 1], ids[5, 3] = E, -(1 << 31)
    ids[6] = [7, 7, 7, 8]                    # the same expert more than once
    logits[7, ids[7]] -= 200                 # chosen ones far below the others
    logits[8] = 1e4 * np.sign(logits[8])
    logits[9] = 0
    dw = rng.normal(size=(T, k)).astype(np.float32).astype(np.float64)
    dd = dw.copy()
    dd[3], dd[4, 1], dd[5, 3] = np.nan, np.nan, np.inf
    dw[3], dw[4, 1], dw[5, 3] = 0, 0, 0
    ref = o.route_grad(logits, ids, dw, renormalize)
    got = grad(logits, ids, dd, renormalize)
    assert np.isfinite(got).all() and not got[0].any() and not got[3].any() and not got[~np.isfinite(logits)].any()
    within(got, ref, bound(logits, ids, dw, renormalize), "dlogits")


@pytest.mark.parametrize("renormalize", [False, True])
def test_against_differences_of_the_router(renormalize):
    """Weights of tl_moe_route at logits +- h: they carry about E half steps of rounding, so the difference quotient is off by
    2 (E + 16) 2^-24 / 2h = 2.7e-4 with h = 2^-6, times |dw|, and by h^2/6 of a third derivative of at most 1 (4.1e-5 |dw|)."""
    T, E, k, h = 40, 20, 3, 2.0 ** -6
    rng = np.random.default_rng(4)
    logits = rng.normal(size=(T, E)).astype(np.float32)
    # chosen ones stay chosen under +- h
    order = np.argsort(-logits, axis=1, kind="stable")
    for t in range(T):
        logits[t, order[t, :k]] += 0.25
    dw = rng.normal(size=(T, k)).astype(np.float32)
    with Lib() as ctx:
        def weights(l):
            ids, w = torch.zeros(T, k, dtype=I32, device="cuda"), torch.zeros(T, k, device="cuda")
            rest = [torch.zeros(n, dtype=I32, device="cuda") for n in (E + 1, T * k, (T * k + E) * 8, 1)]
            tl.tl_moe_route(ctx, gpu(l, F32), T, E, k, renormalize, 128, ids, w, *rest)
            torch.cuda.synchronize()
            by_expert = torch.zeros(T, E, device="cuda", dtype=torch.float64).scatter_(1, ids.long(), w.double())
            return ids, by_expert.cpu().numpy()
        ids, _ = weights(logits)
        ids = ids.cpu().numpy()
        g = np.zeros((T, E))
        np.put_along_axis(g, ids, dw, axis=1)
        num = np.zeros((T, E))
        for i in range(E):
            up, down = logits.copy(), logits.copy()
            up[:, i] += np.float32(h)
            down[:, i] -= np.float32(h)
            num[:, i] = ((weights(up)[1] - weights(down)[1]) * g).sum(1) / (up[:, i].astype(np.float64) - down[:, i])
    got = grad(logits, ids, dw, renormalize)
    within(got, num, (2.7e-4 + 4.1e-5) * np.abs(dw).sum(1, keepdims=True), "dlogits")
