"""Grids of more workgroups than one dimension of a launch takes: every item and row is computed."""
import pytest
import torch

import paper_2503_20313_amd as tl
from oracle import paged as ref
from tests.paged_util import D, HALF_BF16, SCALE, ctx, dev, np64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,T", [(4096, 1024, 1 << 18), (4096, 1024, 4096), (4096, 9, 1 << 18)], ids=str)
def test_every_request_of_a_large_batch(B, H, T):
    """4096 requests at 1024 key heads under 2^18 rows are 1.125 * 2^32 threads.  Rows behind the last token are no memory here: nothing may touch
    them.  All tables list the one page there is; head h's values are h."""
    c = ctx()
    d = tl.tl_paged_dims(batch=B, max_tokens=T, max_new=0, max_blocks=1, page_size=16, n_pages=1, heads_q=H, heads_kv=H, head_dim=D)
    z = tl.tl_paged_query(c, d)
    assert (z["few_items"] + z["tile_items"]) * H > 1 << 16
    if (H, T) == (1024, 1 << 18):
        assert (z["few_items"] + z["tile_items"]) * H * 512 > 1 << 32
    k = torch.ones(H, 16, D, dtype=torch.bfloat16, device=dev())
    v = torch.arange(1, H + 1, device=dev()).to(torch.bfloat16)
    q = torch.zeros(B, H * D, dtype=torch.bfloat16, device=dev())
    o = torch.zeros_like(q)
    zeros = lambda n: torch.zeros(n, dtype=torch.int32, device=dev())      # noqa: E731
    sched, ws = zeros(z["schedule_bytes"] // 4), zeros(z["ws_bytes"] // 4)
    s = torch.cuda.current_stream()
    tl.tl_paged_schedule(c, d, torch.arange(B + 1, dtype=torch.int32, device=dev()), zeros(B) + 16, sched, z["schedule_bytes"], s)
    tl.tl_paged_attention(c, d, q, H * D, k, v[:, None, None].expand(H, 16, D).contiguous(), zeros(B), sched, o, H * D, None, SCALE, ws, z["ws_bytes"], s)
    torch.cuda.synchronize()
    assert int(sched[1]) == B
    assert (o.view(B, H, D) == v[None, :, None]).all()
    tl.tl_ctx_destroy(c)


@pytest.mark.parametrize("T", [(1 << 20) - 1, 1 << 20, (1 << 20) + 1, (1 << 21) + 17], ids=str)
@pytest.mark.parametrize("cached", [False, True], ids=["dense", "cache"])
def test_every_row_of_a_long_step(T, cached):
    """2^20 rows of one query and one key head are 2^16 workgroups; in the cache form (up to 2^18 rows) rows have eight times the heads."""
    Hq, Hk = (1, 1) if not cached else (8, 4)
    T = T if not cached else min(T >> 3, 1 << 18)
    g = torch.Generator(device=dev())
    g.manual_seed(T)
    rows = torch.randn(97, (Hq + 2 * Hk) * D, generator=g, device=dev()).to(torch.bfloat16)
    x = rows.repeat(-(-T // 97), 1)[:T].contiguous()                       # rows repeat every 97
    q, k, v = x.split([Hq * D, Hk * D, Hk * D], 1)
    w = (1 + 0.1 * torch.randn(D, generator=g, device=dev())).to(torch.bfloat16)
    qo, row, c = torch.zeros(T, Hq * D, dtype=torch.bfloat16, device=dev()), x.stride(0), ctx()
    if cached:
        page = 256
        dims = tl.tl_paged_dims(batch=1, max_tokens=T, max_blocks=-(-T // page), page_size=page, n_pages=-(-T // page), heads_q=Hq, heads_kv=Hk, head_dim=D)
        kc, vc = (torch.zeros(dims.n_pages, Hk, page, D, dtype=torch.bfloat16, device=dev()) for _ in range(2))
        tl.tl_qk_norm_rope_cache(c, dims, q, row, k, row, v, row, qo, Hq * D, kc, vc, torch.arange(T, dtype=torch.int32, device=dev()), w, w, 1e-6, None, None, 0, 0,
                                 False, torch.cuda.current_stream())
        ko, vo = (y.transpose(1, 2).reshape(-1, Hk * D)[:T] for y in (kc, vc))
    else:
        ko = torch.zeros(T, Hk * D, dtype=torch.bfloat16, device=dev())
        tl.tl_qk_norm_rope(c, q, row, k, row, qo, Hq * D, ko, Hk * D, T, Hq, Hk, D, w, w, 1e-6, None, None, 0, 0, False, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for got, src, H in ((qo, q, Hq), (ko, k, Hk)):
        y, size = ref.norm_rope(np64(src[:97]).reshape(97, H, D), np64(w), 1e-6, None, None, 0, False)
        err = abs(np64(got[:97]).reshape(97, H, D) - y)
        assert (err <= HALF_BF16 * abs(y) + 2.0 ** -20 * 1.01 * size).all()
        assert torch.equal(got, got[:97].repeat(-(-T // 97), 1)[:T])
    if cached:
        assert torch.equal(vo, v)
    tl.tl_ctx_destroy(c)
