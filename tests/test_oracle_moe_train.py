"""Pins of the mixture-of-experts training oracle: every gradient against differences of the forward definition it belongs to, the
sorted order against a sort with a key, on the CPU."""
import numpy as np
import pytest

from oracle import moe_train as o
from oracle import ops

RNG = np.random.default_rng(250320313)


def differences(f, x, g, h=1e-5):
    """Gradient of <g, f(x)> by central differences: off by O(h^2) and by 1e-16/h of the values, together below 1e-8 here."""
    d = np.zeros(x.shape)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        d[i] = ((f(a) - f(b)) * g).sum() / (2 * h)
    return d


def routing(T, E, k, first=0, local=None):
    ids = np.stack([RNG.permutation(E)[:k] for _ in range(T)])
    return ids, o.sort_rows(ids, first, local or E)


@pytest.mark.parametrize("T,E,k,first,local", [(1, 2, 1, 0, 2), (7, 5, 3, 0, 5), (9, 8, 4, 2, 3), (4, 4, 2, 8, 2)])
def test_sorted_order(T, E, k, first, local):
    ids, (off, order, pos) = routing(T, E, k, first, local)
    mine = [r for r in range(T * k) if first <= ids.flat[r] < first + local]
    assert order.tolist() == sorted(mine, key=lambda r: (ids.flat[r], r))
    assert off[-1] == len(mine) and all(ids.flat[order[s]] - first == e for e in range(local) for s in range(off[e], off[e + 1]))
    assert all(pos.flat[order[s]] == s for s in range(len(order))) and (pos >= 0).sum() == len(order)
    if first == 0 and local == E:
        _, off_ref, rows_ref = ops.moe_sort_rows(ids, E)
        assert np.array_equal(off, off_ref) and np.array_equal(order, rows_ref)


@pytest.mark.parametrize("max_rows", [15, 9])
def test_rows_and_back(max_rows):
    T, H, k = 5, 4, 3
    _, (_, _, pos) = routing(T, 6, k)
    x, w, ys, add = RNG.normal(size=(T, H)), RNG.normal(size=(T, k)), RNG.normal(size=(max_rows, H)), RNG.normal(size=(T, H))
    g_rows, g_tok = RNG.normal(size=(max_rows, H)), RNG.normal(size=(T, H))
    zero = np.zeros((max_rows, H))
    near = dict(rtol=0, atol=1e-8)
    assert np.allclose(o.dispatch_grad(g_rows, pos), differences(lambda a: o.dispatch(a, pos, zero), x, g_rows), **near)
    dys, dw = o.combine_grad(g_tok, ys, w, pos, zero)
    assert np.allclose(dys, differences(lambda a: o.combine(a, w, pos, add), ys, g_tok), **near)
    assert np.allclose(dw, differences(lambda a: o.combine(ys, a, pos, add), w, g_tok), **near)


@pytest.mark.parametrize("renormalize", [False, True])
def test_route_grad(renormalize):
    T, E, k = 6, 7, 3
    ids, _ = routing(T, E, k)
    ids[1, 2] = -1
    ids[2] = E
    logits, dw = RNG.normal(size=(T, E)), RNG.normal(size=(T, k))
    got = o.route_grad(logits, ids, dw, renormalize)
    assert np.allclose(got, differences(lambda a: o.route_weights(a, ids, renormalize), logits, dw), rtol=0, atol=1e-8)
    full = np.argsort(-logits, axis=1, kind="stable")[:, :k]
    _, w_ref = ops.moe_route(logits.astype(np.float32), k, renormalize)
    assert np.allclose(o.route_weights(logits.astype(np.float32).astype(np.float64), full, renormalize), w_ref, rtol=1e-6, atol=1e-7)
    logits[0, :] = -np.inf
    assert not o.route_grad(logits, ids, dw, renormalize)[0].any()


def test_products():
    x, dy, w = RNG.normal(size=(6, 4)), RNG.normal(size=(6, 3)), RNG.normal(size=(3, 4, 3))
    off, add = np.array([0, 2, 2, 6]), RNG.normal(size=(3, 4, 3))
    near = dict(rtol=0, atol=1e-8)
    assert np.allclose(o.products_grad_x(dy, w, off), differences(lambda a: o.products(a, w, off), x, dy), **near)
    assert np.allclose(o.products_grad_w(x, dy, off), differences(lambda a: o.products(x, a, off), w, dy), **near)
    assert np.allclose(o.products_grad_w(x, dy, off, add) - add, o.products_grad_w(x, dy, off))
