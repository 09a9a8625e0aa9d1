"""Harness of the paged-cache tests: a pool of pages in random order with poison everywhere that no token lies, the calls, and
tolerances that follow from the number formats."""
import ctypes

import numpy as np
import torch

import paper_2503_20313_amd as tl
from oracle import paged as ref

D = 128
COUNTERS = 2 * 2 * 2048          # words in front of the workspace's partial results
SCALE = D ** -0.5
HALF_BF16 = torch.finfo(torch.bfloat16).eps / 2       # half a step, relative


def dev():
    return torch.device("cuda", torch.cuda.current_device())


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=dev())


def np64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def ctx():
    return tl.tl_ctx_create(world_size=1, rank=0, channels_per_rank=1, comm_mode=tl.TL_COMM_NONE)


class Batch:
    """Requests with `cached` tokens before and `new` tokens in the step, all of them in the cache."""

    def __init__(self, cached, new, heads_q, heads_kv, page=16, window=0, max_new=None, spare_rows=3, spare_cols=2, spare_pages=3, page_stride=0, seq_lens=None, seed=0,
                 q_std=1.0, cus=None):
        self.g = torch.Generator(device=dev())
        self.g.manual_seed(seed)
        self.page, self.window, self.Hq, self.Hk = page, window, heads_q, heads_kv
        self.new = list(new)
        self.seq = [c + n for c, n in zip(cached, new)] if seq_lens is None else list(seq_lens)
        B, rows = len(self.new), sum(self.new)
        self.T = max(1, rows + spare_rows)
        self.start = np.concatenate([[0], np.cumsum(self.new)])
        need = [-(-s // page) for s in self.seq]
        self.width = max(need + [1]) + spare_cols
        self.n_pages = max(1, sum(need) + spare_pages)
        order = torch.randperm(self.n_pages, generator=self.g, device=dev()).cpu().numpy()
        self.table = np.full((B, self.width), 10 ** 6, np.int64)        # entries that nothing may read: far outside the pool
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        dense = heads_kv * page * D
        self.page_stride = page_stride
        step = page_stride or dense
        pool = [torch.full((self.n_pages * step,), float("nan"), dtype=torch.bfloat16, device=dev()) if step == dense or self.n_pages * step < 1 << 28
                else torch.empty(self.n_pages * step, dtype=torch.bfloat16, device=dev()) for _ in range(2)]
        self.pools = pool
        self.k, self.v = (torch.as_strided(x, (self.n_pages, heads_kv, page, D), (step, page * D, D, 1)) for x in pool)
        for b, s in enumerate(self.seq):
            for j in range(need[b]):
                r = min(page, s - j * page)
                for x in (self.k, self.v):
                    x[int(self.table[b, j]), :, :r] = torch.randn(heads_kv, r, D, generator=self.g, device=dev()).to(torch.bfloat16)
                    x[int(self.table[b, j]), :, r:] = float("nan")
        self.q_stride = heads_q * D + 2 * heads_kv * D                  # rows of a packed projection
        self.qkv = torch.randn(self.T, self.q_stride, generator=self.g, device=dev()).mul_(q_std).to(torch.bfloat16)
        self.qkv[rows:] = float("nan")
        self.o_stride = heads_q * D + 8
        self.rows = rows
        self.dims = tl.tl_paged_dims(batch=B, max_tokens=self.T, max_new=max(self.new + [1]) if max_new is None else max_new, max_blocks=self.width, page_size=page,
                                     n_pages=self.n_pages, heads_q=heads_q, heads_kv=heads_kv, head_dim=D, window=window, page_stride=page_stride)

    def reference(self):
        q = np64(self.qkv[:, :self.Hq * D]).reshape(self.T, self.Hq, D)
        return ref.attention(q, np64(self.k), np64(self.v), self.table, self.start, self.seq, self.page, self.window, SCALE)

    def buffers(self, c):
        z = tl.tl_paged_query(c, self.dims)
        self.ws_bytes, self.sched_bytes = z["ws_bytes"], z["schedule_bytes"]
        self.ws = torch.zeros(self.ws_bytes // 4, device=dev())
        self.ws[COUNTERS:] = float("nan")                                   # of the partial results nothing is needed before they are written
        self.schedule = torch.full((self.sched_bytes // 4,), -1, dtype=torch.int32, device=dev())
        self.o = torch.full((self.T, self.o_stride), 7.0, dtype=torch.bfloat16, device=dev())
        self.lse = torch.full((self.T, self.Hq), 7.0, device=dev())
        self.start_d, self.seq_d, self.table_d = ints(self.start), ints(self.seq), ints(self.table)
        return z

    def schedule_call(self, c, stream=None):
        tl.tl_paged_schedule(c, self.dims, self.start_d, self.seq_d, self.schedule, self.sched_bytes, stream)

    def attention_call(self, c, stream=None, lse=True):
        tl.tl_paged_attention(c, self.dims, self.qkv, self.q_stride, self.pools[0], self.pools[1], self.table_d, self.schedule, self.o, self.o_stride,
                              self.lse if lse else None, SCALE, self.ws, self.ws_bytes, stream)

    def run(self, lse=True):
        c = ctx()
        self.buffers(c)
        s = torch.cuda.current_stream()
        self.schedule_call(c, s)
        self.attention_call(c, s, lse)
        torch.cuda.synchronize()
        tl.tl_ctx_destroy(c)
        assert not self.ws[:COUNTERS].view(torch.int32).any(), "a counter is not back at zero"
        return self.o, self.lse


def check_attention(b, want=None, lse=True):
    """o: its own rounding, the rounding of the probabilities (relative to the sum of their absolute terms), and the fp32 scores:
    a score is a sum of 128 products of size scale*|q||k| (about 7 in all for unit normal inputs), off by at most 130 * 2^-24 of
    that, and the exponents of numerator and denominator differ by twice it: under 2^-12.  lse: that and its fp32 sum: 2^-11."""
    o_ref, lse_ref, size = b.reference() if want is None else want
    n = b.rows
    o = np64(b.o[:n, :b.Hq * D]).reshape(n, b.Hq, D)
    tol = 1.01 * (HALF_BF16 * np.abs(o_ref[:n]) + (HALF_BF16 + 2.0 ** -12) * size[:n]) + 1e-30
    fin = np.isfinite(o_ref[:n])
    bad = np.abs(o[fin] - o_ref[:n][fin]) > tol[fin]
    assert not np.isnan(o[fin]).any(), f"{np.isnan(o[fin]).sum()} NaN where the result is finite"
    assert not bad.any(), f"{bad.sum()} of {bad.size} elements off, worst {np.max(np.abs(o[fin] - o_ref[:n][fin]) / tol[fin]):.2f} of the tolerance"
    same = np.where(np.isnan(o_ref[:n]), np.isnan(o), o == o_ref[:n])
    assert same[~fin].all(), "non-finite results differ"
    if lse:
        got, w = np64(b.lse[:n]), lse_ref[:n]
        f = np.isfinite(w)
        assert (np.abs(got[f] - w[f]) <= 2.0 ** -11 + 2.0 ** -22 * np.abs(w[f])).all(), np.max(np.abs(got[f] - w[f]))
        assert (got[~f] == w[~f])[~np.isnan(w[~f])].all()
    # nothing else was written
    assert (b.o[n:] == 7).all() and (b.o[:, b.Hq * D:] == 7).all() and (b.lse[n:] == 7).all()


def as_c(dims):
    return ctypes.byref(dims)
