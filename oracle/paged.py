"""Plain CPU definitions of the paged-cache operators (test infrastructure only): float64 numpy, nothing rounded."""
from __future__ import annotations

import math

import numpy as np


def slots(ctx_lens, new_lens, free_pages, free_from, block_table, T, max_new, page, n_pages):
    """What tl_paged_slots writes, request by request and token by token."""
    table = np.array(block_table, copy=True)
    width = table.shape[1]
    cap = width * page
    out_slots, positions = np.full(T, -1, np.int64), np.zeros(T, np.int64)
    start, seq = [0], []
    used, lacking, over, row = 0, 0, 0, 0
    for b, (c, n) in enumerate(zip(ctx_lens, new_lens)):
        c, want = min(max(int(c), 0), cap), max(int(n), 0)
        n = min(want, max_new, cap - c, T - row)
        over += want - n
        for j in range(-(-c // page), -(-(c + n) // page)):
            i = free_from + used + lacking
            if i < len(free_pages):
                table[b, j] = free_pages[i]
                used += 1
            else:
                table[b, j] = -1
                lacking += 1
        for i in range(n):
            p = table[b, (c + i) // page]
            out_slots[row + i] = p * page + (c + i) % page if 0 <= p < n_pages else -1
            positions[row + i] = c + i
        row += n
        start.append(row)
        seq.append(c + n)
    return dict(table=table, query_start=np.array(start), seq_lens=np.array(seq), slots=out_slots, positions=positions, free_to=free_from + used,
                counts=np.array([row, used, lacking, min(over, 2 ** 31 - 1)]))


def norm_rope(x, weight, eps, positions, cos_sin, rot, interleaved):
    """x [T, heads, D] float64 -> the normed and rotated heads, and the size of the terms every element is made of."""
    x = np.array(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    y, size = x.copy(), np.abs(x)
    for t in range(x.shape[0]):
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
            c, s = cos_sin[positions[t], i], cos_sin[positions[t], rot // 2 + i]
            y[t, :, a], y[t, :, b] = x[t, :, a] * c - x[t, :, b] * s, x[t, :, b] * c + x[t, :, a] * s
            size[t, :, a] = size[t, :, b] = np.abs(x[t, :, a]) + np.abs(x[t, :, b])
    return y, size


def attention(q, k_cache, v_cache, table, query_start, seq_lens, page, window, scale):
    """q [T, Hq, D], caches [n_pages, Hk, page, D], float64.  Every row sums over the keys it sees, and over those alone.
    Returns o [T, Hq, D], lse [T, Hq], and size = sum_j p_j |v_j| (what the rounding of the probabilities goes by).  Rows of no
    request stay NaN."""
    T, Hq, D = q.shape
    n_pages, Hk = k_cache.shape[:2]
    G = Hq // Hk
    o, lse, size = np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan), np.full((T, Hq, D), np.nan)
    for b, seq in enumerate(seq_lens):
        r0, n = query_start[b], query_start[b + 1] - query_start[b]
        if n <= 0:
            continue
        key = np.arange(seq)
        pg = table[b, key // page]
        real = (pg >= 0) & (pg < n_pages)
        for h in range(Hk):
            k = np.zeros((seq, D))
            v = np.zeros((seq, D))
            k[real], v[real] = k_cache[pg[real], h, key[real] % page], v_cache[pg[real], h, key[real] % page]
            for i in range(n):
                pos = seq - n + i
                seen = np.nonzero(real & (key <= pos) & (key > pos - window if window else True))[0]
                for hq in range(h * G, (h + 1) * G):
                    if len(seen) == 0:
                        o[r0 + i, hq], lse[r0 + i, hq], size[r0 + i, hq] = 0, -math.inf, 0
                        continue
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = k[seen] @ q[r0 + i, hq] * scale
                        m = s.max()
                        p = np.exp(s - m)
                        l = p.sum()
                        o[r0 + i, hq], size[r0 + i, hq] = p @ v[seen] / l, p @ np.abs(v[seen]) / l
                        lse[r0 + i, hq] = m + math.log(l) if l == l else math.nan
    return o, lse, size
