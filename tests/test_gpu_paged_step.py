"""The paged-cache operators as a serving loop uses them: with the framework's own projections around them, captured, and
against an attention that keeps every token's key and value in a list."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from oracle import paged as ref
from tests.paged_util import D, HALF_BF16, SCALE, ctx, dev, ints, np64

pytestmark = pytest.mark.gpu
EPS, ROT, MAXPOS = 1e-6, 128, 512


def angles():
    f = 10000.0 ** (-np.arange(0, ROT, 2) / ROT)
    a = np.arange(MAXPOS)[:, None] * f
    return torch.tensor(np.concatenate([np.cos(a), np.sin(a)], 1), dtype=torch.float32, device=dev())


class Layer:
    """One rank's share of an attention layer of R ranks: packed projection (AllGather + GEMM), the paged operators, and the output
    projection (GEMM + ReduceScatter)."""

    def __init__(self, T, R, Hq, Hk, H, B, page, width, n_pages, max_new, window):
        g = torch.Generator(device=dev())
        g.manual_seed(7)
        self.T, self.R, self.Hq, self.Hk, self.H = T, R, Hq, Hk, H
        N = (Hq + 2 * Hk) * D

        def normal(*shape, std=1.0):
            return torch.randn(shape, generator=g, device=dev()).mul_(std).to(torch.bfloat16)
        self.normal = normal
        self.w_in, self.w_out = normal(H, N, std=0.05), normal(Hq * D, H, std=0.02)
        self.wq, self.wk = (normal(D, std=0.1) + 1 for _ in range(2))
        self.cs = angles()
        kw = dict(world_size=R, rank=1, channels_per_rank=1, comm_mode=tl.TL_COMM_SIDE_KERNEL, tile_order=tl.TL_ORDER_OWN_FIRST, xcd_swizzle=1,
                  spin_timeout_us=5_000_000)
        self.c1, self.c2, self.c = tl.tl_ctx_create(**kw), tl.tl_ctx_create(rs_direct_push=1, **kw), ctx()
        zeros = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device=dev())
        bf = torch.bfloat16
        (self.ws1, f1), (self.ws2, f2) = tl.tl_query_workspace(self.c1, tl.TL_OP_AG_GEMM, [T, N, H]), tl.tl_query_workspace(self.c2, tl.TL_OP_GEMM_RS, [T, H, Hq * D])
        self.flags1, self.flags2, self.w1, self.w2 = zeros(f1), zeros(f2), zeros(self.ws1 // 4), zeros(self.ws2 // 4)
        self.epoch = 0
        self.x, self.qkv = zeros(T, H, dtype=bf), zeros(T, N, dtype=bf)
        self.shards = [zeros(T // R, H, dtype=bf) for _ in range(R)]
        self.partial, self.out = zeros(T, H, dtype=bf), zeros(T // R, H, dtype=bf)
        self.recv = [0 if q == 1 else zeros(T // R, H, dtype=bf) for q in range(R)]
        self.push = [0 if q == 1 else zeros(T // R, H, dtype=bf) for q in range(R)]
        self.q, self.o = zeros(T, Hq * D, dtype=bf), zeros(T, Hq * D, dtype=bf)
        self.kc, self.vc = (torch.full((n_pages, Hk, page, D), float("nan"), dtype=bf, device=dev()) for _ in range(2))
        self.dims = tl.tl_paged_dims(batch=B, max_tokens=T, max_new=max_new, max_blocks=width, page_size=page, n_pages=n_pages, heads_q=Hq, heads_kv=Hk, head_dim=D,
                                     window=window)
        z = tl.tl_paged_query(self.c, self.dims)
        self.schedule, self.ws, self.sb, self.wb = zeros(z["schedule_bytes"] // 4), zeros(z["ws_bytes"] // 4), z["schedule_bytes"], z["ws_bytes"]
        self.lens, self.new, self.frm = zeros(B), zeros(B), zeros(1)
        self.free = torch.randperm(n_pages, generator=g, device=dev()).to(torch.int32)
        self.table = torch.full((B, width), -9, dtype=torch.int32, device=dev())
        self.qs, self.slots, self.pos, self.counts = zeros(B + 1), zeros(T), zeros(T), zeros(4)
        self.comm = torch.cuda.Stream()

    def paged(self):
        s = torch.cuda.current_stream()
        row, d = self.qkv.stride(0), self.dims
        q, k, v = self.qkv.split([self.Hq * D, self.Hk * D, self.Hk * D], 1)
        tl.tl_paged_slots(self.c, d, self.lens, self.new, self.free, self.free.numel(), self.frm, self.frm, self.table, self.qs, self.lens, self.slots, self.pos,
                          self.counts, s)
        tl.tl_paged_schedule(self.c, d, self.qs, self.lens, self.schedule, self.sb, s)
        tl.tl_qk_norm_rope_cache(self.c, d, q, row, k, row, v, row, self.q, self.Hq * D, self.kc, self.vc, self.slots, self.wq, self.wk, EPS, self.pos, self.cs,
                                 MAXPOS, ROT, False, s)
        tl.tl_paged_attention(self.c, d, self.q, self.Hq * D, self.kc, self.vc, self.table, self.schedule, self.o, self.Hq * D, None, SCALE, self.ws, self.wb, s)

    def step(self, graph):
        cs, T, N = torch.cuda.current_stream(), self.T, self.qkv.shape[1]
        self.epoch += 1
        self.comm.wait_stream(cs)
        tl.tl_ag_gemm(self.c1, self.shards, self.x, self.w_in, self.qkv, T, N, self.H, self.flags1, self.epoch, self.w1, self.ws1, cs, self.comm)
        cs.wait_stream(self.comm)
        graph.replay()
        self.comm.wait_stream(cs)
        tl.tl_gemm_rs(self.c2, self.o, self.w_out, self.partial, self.recv, self.push, self.out, T, self.H, self.Hq * D, self.flags2, self.epoch, self.w2, self.ws2,
                      cs, self.comm)
        torch.cuda.synchronize()
        tl.tl_check_status(self.c1, self.w1)
        tl.tl_check_status(self.c2, self.w2)

    def close(self):
        for c in (self.c, self.c1, self.c2):
            tl.tl_ctx_destroy(c)


@pytest.mark.parametrize("window", [0, 40])
def test_serving_loop(window):
    """Prompts of several lengths, then tokens one by one, then another prompt beside them; the paged part is one graph.  The
    reference keeps the rounded keys and values that the layer's own projection gives and attends to them in 64 bits."""
    T, R, Hq, Hk, H, B = 128, 2, 6, 2, 512, 5
    L = Layer(T, R, Hq, Hk, H, B, page=16, width=12, n_pages=40, max_new=90, window=window)
    L.o.fill_(3)
    warm = torch.cuda.Stream()
    with torch.cuda.stream(warm):      # (nothing is new yet: the calls run and write nothing)
        L.paged()
    torch.cuda.synchronize()
    assert (L.o == 3).all() and L.counts.tolist() == [0, 0, 0, 0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.paged()
    cs, wq, wk = np64(L.cs), np64(L.wq), np64(L.wk)
    seen = [([], []) for _ in range(B)]
    for new in ([17, 0, 33, 1, 0], [1, 0, 1, 1, 0], [1, 0, 1, 1, 0], [1, 70, 1, 1, 5], [2, 1, 0, 1, 1], [1, 1, 1, 1, 1]):
        L.new.copy_(ints(new))
        for x in L.shards:
            x.copy_(L.normal(T // R, H))
        L.o.fill_(3)
        L.step(g)
        n = sum(new)
        assert L.counts.tolist() == [n, L.counts[1].item(), 0, 0]
        got_q, qkv, o = np64(L.q).reshape(T, Hq, D), np64(L.qkv), np64(L.o).reshape(T, Hq, D)
        assert (o[n:] == 3).all()
        row = 0
        for b, m in enumerate(new):
            at = len(seen[b][0])
            pos = np.arange(at, at + m)
            xq, xk, xv = np.split(qkv[row:row + m], [Hq * D, (Hq + Hk) * D], 1)
            yq, sq = ref.norm_rope(xq.reshape(m, Hq, D), wq, EPS, pos, cs, ROT, False)
            yk, sk = ref.norm_rope(xk.reshape(m, Hk, D), wk, EPS, pos, cs, ROT, False)
            assert (np.abs(got_q[row:row + m] - yq) <= HALF_BF16 * np.abs(yq) + 2.0 ** -20 * 1.01 * sq).all()
            # the cache's own rounded keys, checked and then used
            for i in range(m):
                slot = int(L.slots[row + i])
                k = np64(L.kc[slot // 16, :, slot % 16])
                assert (np.abs(k - yk[i]) <= HALF_BF16 * np.abs(yk[i]) + 2.0 ** -20 * 1.01 * sk[i]).all()
                assert np.array_equal(np64(L.vc[slot // 16, :, slot % 16]), xv[i].reshape(Hk, D))
                seen[b][0].append(k)
                seen[b][1].append(xv[i].reshape(Hk, D))
            for i in range(m):
                lo = max(0, at + i + 1 - window) if window else 0
                K, V = (np.stack(x[lo:at + i + 1]) for x in seen[b])
                for h in range(Hq):
                    s = K[:, h // (Hq // Hk)] @ got_q[row + i, h] * SCALE
                    p = np.exp(s - s.max())
                    want, size = p @ V[:, h // (Hq // Hk)] / p.sum(), p @ np.abs(V[:, h // (Hq // Hk)]) / p.sum()
                    # as for the attention alone; its queries and keys are normed here: their products are at most 128 * 1.5^2 * scale = 26
                    assert (np.abs(o[row + i, h] - want) <= 1.01 * (HALF_BF16 * np.abs(want) + (HALF_BF16 + 2.0 ** -11) * size)).all()
            row += m
        assert [len(s[0]) for s in seen] == L.lens.tolist()
        # the output projection reads those rows
        own = np64(L.partial[T // R:])
        want = np64(L.o)[T // R:] @ np64(L.w_out)
        size = np.abs(np64(L.o))[T // R:] @ np.abs(np64(L.w_out))
        assert (np.abs(own - want) <= HALF_BF16 * np.abs(want) + Hq * D * 2.0 ** -24 * size).all()
    L.close()


def test_norm_and_rotation_before_the_sequence_parallel_attention():
    """tl_qk_norm_rope on the local shards of queries and keys, then tl_sp_ag_attention over all ranks' shards."""
    S, heads, R, rank = 512, 4, 2, 1
    n = S // R
    g = torch.Generator(device=dev())
    g.manual_seed(9)
    q, k, v = (torch.randn(S, heads * D, generator=g, device=dev()).to(torch.bfloat16) for _ in range(3))
    wq, wk = (torch.randn(D, generator=g, device=dev()).mul_(0.1).add_(1).to(torch.bfloat16) for _ in range(2))
    cs, c, row = angles(), ctx(), heads * D
    rq, rk = torch.empty_like(q), torch.empty_like(k)
    for r in range(R):                     # every rank does this for its own rows
        a = slice(r * n, (r + 1) * n)
        tl.tl_qk_norm_rope(c, q[a], row, k[a], row, rq[a], row, rk[a], row, n, heads, heads, D, wq, wk, EPS, torch.arange(r * n, (r + 1) * n, dtype=torch.int32, device=dev()),
                           cs, MAXPOS, ROT, False, torch.cuda.current_stream())
    sp = tl.tl_ctx_create(world_size=R, rank=rank, channels_per_rank=1, comm_mode=tl.TL_COMM_WAVES, spin_timeout_us=5_000_000)
    info = tl.tl_attn_query(sp, S, heads, D, True)
    kg, vg, o = torch.zeros_like(k), torch.zeros_like(v), torch.zeros(n, row, dtype=torch.bfloat16, device=dev())
    flags, ws = torch.zeros(info["n_flags"], dtype=torch.int32, device=dev()), torch.zeros(info["ws_bytes"] // 4, dtype=torch.int32, device=dev())
    s = torch.cuda.current_stream()
    tl.tl_sp_ag_attention(sp, rq[rank * n:], [rk[:n], rk[n:]], [v[:n], v[n:]], kg, vg, o, S, heads, D, True, SCALE, flags, 1, ws, info["ws_bytes"], s, s)
    torch.cuda.synchronize()
    tl.tl_check_status(sp, ws)
    yq, _ = ref.norm_rope(np64(q).reshape(S, heads, D), np64(wq), EPS, np.arange(S), np64(cs), ROT, False)
    yk, _ = ref.norm_rope(np64(k).reshape(S, heads, D), np64(wk), EPS, np.arange(S), np64(cs), ROT, False)
    got, V = np64(o).reshape(n, heads, D), np64(v).reshape(S, heads, D)
    for h in range(heads):
        x = yq[rank * n:, h] @ yk[:, h].T * SCALE
        x[np.arange(S)[None] > np.arange(rank * n, S)[:, None]] = -np.inf
        p = np.exp(x - x.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        want, size = p @ V[:, h], p @ np.abs(V[:, h])
        # queries and keys are rounded: a score moves by at most 2 * 2^-8 of sum |q||k| * scale <= 128 * 1.5^2 * scale = 26, by sqrt(128) less in
        # the norm; taken as 2^-7 * 26 / 8, both ways of the quotient
        assert (np.abs(got[:, h] - want) <= 1.01 * (HALF_BF16 * np.abs(want) + (HALF_BF16 + 2 * 2.0 ** -7 * 26 / 8) * size)).all()
    tl.tl_ctx_destroy(c)
    tl.tl_ctx_destroy(sp)
