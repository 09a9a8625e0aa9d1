"""Plain CPU definitions of a mixture-of-experts layer's parts in training (test infrastructure only), in float64 numpy.  Tensors are
float64 arrays of the values the device holds; nothing is rounded here."""
from __future__ import annotations

import numpy as np


def sort_rows(ids, first, E):
    """Rows (t, j) = t*topk + j whose expert is in [first, first + E), by (expert, row): offsets [E+1], rows in that order, and
    every row's place or -1."""
    flat = np.asarray(ids, np.int64).reshape(-1) - first
    order = [r for e in range(E) for r in np.nonzero(flat == e)[0]]
    offsets = np.concatenate([[0], np.cumsum([(flat == e).sum() for e in range(E)])]).astype(np.int64)
    pos = np.full(flat.shape, -1, np.int64)
    pos[np.array(order, np.int64)] = np.arange(len(order))
    return offsets, np.array(order, np.int64), pos.reshape(np.shape(ids))


def _places(row_pos, max_rows):
    """(t, j, place) of the rows that take part, in the order of j inside a token."""
    for t, j in np.ndindex(*row_pos.shape):
        if 0 <= row_pos[t, j] < max_rows:
            yield t, j, int(row_pos[t, j])


def dispatch(x, row_pos, xs):
    out = xs.copy()
    for t, _, at in _places(row_pos, len(xs)):
        out[at] = x[t]
    return out


def dispatch_grad(dxs, row_pos):
    dx = np.zeros((row_pos.shape[0], dxs.shape[1]))
    for t, _, at in _places(row_pos, len(dxs)):
        dx[t] += dxs[at]
    return dx


def combine(ys, w, row_pos, add=None):
    out = np.zeros((row_pos.shape[0], ys.shape[1])) if add is None else add.copy()
    for t, j, at in _places(row_pos, len(ys)):
        out[t] += w[t, j] * ys[at]
    return out


def combine_grad(dout, ys, w, row_pos, dys):
    dys, dw = dys.copy(), np.zeros(row_pos.shape)
    for t, j, at in _places(row_pos, len(ys)):
        dw[t, j] = dout[t] @ ys[at]
    for t, j, at in _places(row_pos, len(ys)):
        dys[at] = w[t, j] * dout[t]
    return dys, dw


def route_weights(logits, ids, renormalize):
    """Weights of the listed experts; an id that is none has no weight."""
    w = np.zeros(ids.shape)
    for t in range(len(logits)):
        real = (ids[t] >= 0) & (ids[t] < logits.shape[1])
        chosen = logits[t][ids[t][real]]
        among = chosen if renormalize else logits[t]
        if among.size and among.max() > -np.inf:
            w[t, real] = np.exp(chosen - among.max()) / np.exp(among - among.max()).sum()
    return w


def route_grad(logits, ids, dw, renormalize):
    """Row by row through the Jacobian of the weights: d w_j / d l_i = w_j ([i = e_j] - q_i), q_i = the share of i among what w_j is
    normalised over."""
    w = route_weights(logits, ids, renormalize)
    out = np.zeros(logits.shape)
    for t in range(len(logits)):
        real = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < logits.shape[1]]
        share = np.zeros(logits.shape[1])
        if renormalize:
            for j in real:
                share[ids[t, j]] += w[t, j]
        elif logits[t].max() > -np.inf:
            share = np.exp(logits[t] - logits[t].max())
            share /= share.sum()
        for j in real:
            if w[t, j] == 0:
                continue
            d = -share
            d[ids[t, j]] += 1.0
            out[t] += dw[t, j] * w[t, j] * d
    return out


def products(x, w, offsets):
    """Y, rows beyond the experts' as NaN."""
    y = np.full((len(x), w.shape[2]), np.nan)
    for e in range(len(w)):
        y[offsets[e]:offsets[e + 1]] = x[offsets[e]:offsets[e + 1]] @ w[e]
    return y


def products_grad_x(dy, w, offsets):
    return products(dy, w.transpose(0, 2, 1), offsets)


def products_grad_w(x, dy, offsets, add=None):
    E = len(offsets) - 1
    dw = np.zeros((E, x.shape[1], dy.shape[1])) if add is None else add.copy()
    for e in range(E):
        dw[e] += x[offsets[e]:offsets[e + 1]].T @ dy[offsets[e]:offsets[e + 1]]
    return dw
