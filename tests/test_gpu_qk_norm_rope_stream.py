"""tl_qk_norm_rope_cache with results larger than the dies' caches together, which are stored as streaming."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from tests.paged_util import D, ctx, dev
from tests.test_gpu_qk_norm_rope import EPS, MAXPOS, angles, close, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,Hq,Hk,page,rot,inter,norm", [(8001, 32, 8, 64, 64, False, True), (2500, 40, 10, 16, 128, True, True), (40000, 3, 1, 256, 48, False, False)], ids=str)
def test_large_results_into_the_cache(T, Hq, Hk, page, rot, inter, norm):
    """Random slots, some rows of padding, some rows without a position, pages that lie apart; slots of no row stay as they were."""
    assert T * (Hq + 2 * Hk) * D * 2 > 32 << 20
    qkv, w, pos = draw(T, Hq, Hk, 71, pad=8)
    wq, wk = w if norm else (None, None)
    cs, row = angles(rot), qkv.stride(0)
    n_pages, step = -(-T // page) + 5, page * Hk * D + 64
    pools = [torch.full((n_pages * step,), 7.0, dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(72))[:T].to(torch.int32)
    slots[::101], slots[5], slots[T - 1] = -1, n_pages * page, -(1 << 31)
    pos[7::997] = -1
    pos[8] = MAXPOS
    qo = torch.full((T, Hq * D + 8), 7.0, dtype=torch.bfloat16, device=dev())
    dims = tl.tl_paged_dims(batch=1, max_tokens=T, max_blocks=n_pages, page_size=page, n_pages=n_pages, heads_q=Hq, heads_kv=Hk, head_dim=D, page_stride=step)
    q, k, v = qkv.split([Hq * D, Hk * D, Hk * D + 8], 1)
    c = ctx()
    tl.tl_qk_norm_rope_cache(c, dims, q, row, k, row, v, row, qo, Hq * D + 8, *pools, slots.to(dev()), wq, wk, EPS, pos, cs, MAXPOS, rot, inter,
                             torch.cuda.current_stream())
    torch.cuda.synchronize()
    tl.tl_ctx_destroy(c)
    s, p = slots.long(), pos.cpu()
    keep = (s >= 0) & (s < n_pages * page) & (p >= 0) & (p < MAXPOS)
    kc, vc = (torch.as_strided(x, (n_pages, Hk, page, D), (step, page * D, D, 1)) for x in pools)
    kd, at = keep.to(dev()), s[keep].to(dev())
    vals = vc[at // page, :, at % page].reshape(-1, Hk * D)
    assert torch.equal(vals, v[kd][:, :Hk * D])
    assert (qo[~kd] == 7).all() and (qo[:, Hq * D:] == 7).all()
    used = torch.zeros(n_pages * page, dtype=torch.bool, device=dev())
    used[at] = True
    for x, pool in ((kc, pools[0]), (vc, pools[1])):
        flat = x.transpose(1, 2).reshape(n_pages * page, Hk * D)
        assert (flat[~used] == 7).all() and (flat[used] != 7).any(1).all()
        assert (pool.view(n_pages, step)[:, Hk * page * D:] == 7).all()
    # rows all over the call, against the definition
    some = np.unique(np.concatenate([[0, 1, 2, 15, 16, T // 2, T - 3, T - 2], np.random.default_rng(73).integers(0, T, 60)]))
    some = torch.from_numpy(some)[keep[some]]
    sd, pn = some.to(dev()), p[some].numpy()
    close(qo[sd][:, :Hq * D], q[sd], Hq, wq, pn, cs, rot, inter)
    ks = s[some].to(dev())
    close(kc[ks // page, :, ks % page].reshape(-1, Hk * D), k[sd], Hk, wk, pn, cs, rot, inter)
