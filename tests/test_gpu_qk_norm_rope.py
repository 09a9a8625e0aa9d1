"""tl_qk_norm_rope and tl_qk_norm_rope_cache against the plain definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from oracle import paged as ref
from tests.paged_util import D, HALF_BF16, ctx, dev, ints, np64

pytestmark = pytest.mark.gpu
EPS = 1e-6
MAXPOS = 300


def angles(rot, n=MAXPOS):
    f = 10000.0 ** (-np.arange(0, max(rot, 2), 2) / max(rot, 1))[:max(rot // 2, 1)]
    a = np.arange(n)[:, None] * f
    return torch.tensor(np.concatenate([np.cos(a), np.sin(a)], 1), dtype=torch.float32, device=dev())


def draw(T, Hq, Hk, seed, pad=0):
    g = torch.Generator(device=dev())
    g.manual_seed(seed)
    qkv = torch.randn(T, (Hq + 2 * Hk) * D + pad, generator=g, device=dev()).to(torch.bfloat16)
    w = [(1 + 0.2 * torch.randn(D, generator=g, device=dev())).to(torch.bfloat16) for _ in range(2)]
    return qkv, w, torch.randint(0, MAXPOS, (T,), generator=g, device=dev(), dtype=torch.int32)


def close(got, x, heads, w, pos, cs, rot, inter, keep=None):
    """Half a step of the result, and of its terms 2^-20: 12 roundings in the mean of squares (half of them reach the root), the root, the
    quotient, two products, and three in the rotation, of 2^-24 each."""
    T = x.shape[0]
    y, size = ref.norm_rope(np64(x).reshape(T, heads, D), None if w is None else np64(w), EPS, pos, np64(cs), rot, inter)
    err = np.abs(np64(got).reshape(T, heads, D) - y)
    ok = err <= HALF_BF16 * np.abs(y) + 2.0 ** -20 * size * 1.01
    if keep is not None:
        ok = ok[keep]
    assert ok.all(), f"{(~ok).sum()} of {ok.size} off"


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("rot", [0, 16, 48, 64, 128])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("shape", [(1, 32, 8), (5, 3, 1), (70, 1, 1)], ids=str)
def test_rows(shape, rot, norm, inter):
    T, Hq, Hk = shape
    qkv, w, pos = draw(T, Hq, Hk, 1)
    cs = angles(rot)
    wq, wk = w if norm else (None, None)
    qo = torch.full((T, Hq * D + 8), 7.0, dtype=torch.bfloat16, device=dev())
    ko = torch.full((T, Hk * D + 16), 7.0, dtype=torch.bfloat16, device=dev())
    c = ctx()
    row = qkv.stride(0)
    q, k = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D]
    tl.tl_qk_norm_rope(c, q, row, k, row, qo, qo.stride(0), ko, ko.stride(0), T, Hq, Hk, D, wq, wk, EPS, pos if rot else None, cs if rot else None,
                       MAXPOS if rot else 0, rot, inter, torch.cuda.current_stream())
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    close(qo[:, :Hq * D], q, Hq, wq, p, cs, rot, inter)
    close(ko[:, :Hk * D], k, Hk, wk, p, cs, rot, inter)
    assert (qo[:, Hq * D:] == 7).all() and (ko[:, Hk * D:] == 7).all()
    if not norm and rot == 0:
        assert torch.equal(qo[:, :Hq * D], q)
    tl.tl_ctx_destroy(c)


def test_in_place_and_rows_without_a_position():
    T, Hq, Hk, rot = 40, 4, 2, 64
    qkv, (wq, wk), pos = draw(T, Hq, Hk, 2)
    pos[3], pos[17], pos[39] = -1, MAXPOS, 2 ** 31 - 1
    cs, before, row = angles(rot), qkv.clone(), qkv.stride(0)
    q, k = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D]
    c = ctx()
    tl.tl_qk_norm_rope(c, q, row, k, row, q, row, k, row, T, Hq, Hk, D, wq, wk, EPS, pos, cs, MAXPOS, rot, False)
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    keep = (p >= 0) & (p < MAXPOS)
    p = np.where(keep, p, 0)
    close(qkv[:, :Hq * D], before[:, :Hq * D], Hq, wq, p, cs, rot, False, keep)
    close(qkv[:, Hq * D:(Hq + Hk) * D], before[:, Hq * D:(Hq + Hk) * D], Hk, wk, p, cs, rot, False, keep)
    out = torch.from_numpy(~keep).to(dev())
    assert torch.equal(qkv[out], before[out]) and torch.equal(qkv[:, (Hq + Hk) * D:], before[:, (Hq + Hk) * D:])
    tl.tl_ctx_destroy(c)


def test_results_larger_than_the_caches():
    """Streaming stores; the first and last rows and some between are compared."""
    T, Hq, Hk = 9001, 16, 4
    qkv, (wq, wk), pos = draw(T, Hq, Hk, 8)
    cs, row = angles(128), qkv.stride(0)
    qo, ko = torch.zeros(T, Hq * D, dtype=torch.bfloat16, device=dev()), torch.zeros(T, Hk * D, dtype=torch.bfloat16, device=dev())
    c = ctx()
    q, k = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D]
    tl.tl_qk_norm_rope(c, q, row, k, row, qo, Hq * D, ko, Hk * D, T, Hq, Hk, D, wq, wk, EPS, pos, cs, MAXPOS, 128, False)
    torch.cuda.synchronize()
    some = torch.tensor([0, 1, 15, 16, 4000, 8191, 8192, T - 2, T - 1], device=dev())
    p = pos[some].cpu().numpy()
    close(qo[some], q[some], Hq, wq, p, cs, 128, False)
    close(ko[some], k[some], Hk, wk, p, cs, 128, False)
    assert (qo != 0).any(1).all() and (ko != 0).any(1).all()
    tl.tl_ctx_destroy(c)


def test_zero_rows_and_large_values():
    """A row of zeros is finite (eps); values whose squares leave the range of bf16 but not of fp32 are normed alike."""
    T, Hq, Hk = 3, 2, 1
    qkv, (wq, wk), pos = draw(T, Hq, Hk, 3)
    qkv[0] = 0
    qkv[1] *= 2.0 ** 50
    qkv[2] *= 2.0 ** -5
    cs, row = angles(128), qkv.stride(0)
    qo, ko = torch.zeros(T, Hq * D, dtype=torch.bfloat16, device=dev()), torch.zeros(T, Hk * D, dtype=torch.bfloat16, device=dev())
    c = ctx()
    q, k = qkv[:, :Hq * D], qkv[:, Hq * D:(Hq + Hk) * D]
    tl.tl_qk_norm_rope(c, q, row, k, row, qo, Hq * D, ko, Hk * D, T, Hq, Hk, D, wq, wk, EPS, pos, cs, MAXPOS, 128, False)
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    close(qo, q, Hq, wq, p, cs, 128, False)
    close(ko, k, Hk, wk, p, cs, 128, False)
    assert (qo[0] == 0).all()
    tl.tl_ctx_destroy(c)


@pytest.mark.parametrize("page,stride", [(16, 0), (64, 64 * 2 * D + 128)])
@pytest.mark.parametrize("shape", [(1, 8, 1), (33, 4, 2), (200, 10, 2)], ids=str)
def test_into_the_cache(shape, page, stride):
    T, Hq, Hk = shape
    if stride:
        stride = page * Hk * D + 128
    qkv, (wq, wk), pos = draw(T, Hq, Hk, 4, pad=16)
    rot, cs, row = 128, angles(128), qkv.stride(0)
    n_pages = -(-T // page) + 3
    step = stride or page * Hk * D
    pools = [torch.full((n_pages * step,), 7.0, dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(5))[:T].to(torch.int32)
    pad = [i for i in (0, T // 2, T - 1) if T > 3]
    for i, x in zip(pad, (-1, n_pages * page, -(1 << 31))):
        slots[i] = x
    qo = torch.full((T, Hq * D), 7.0, dtype=torch.bfloat16, device=dev())
    dims = tl.tl_paged_dims(batch=1, max_tokens=T, max_blocks=n_pages, page_size=page, n_pages=n_pages, heads_q=Hq, heads_kv=Hk, head_dim=D, page_stride=stride)
    c = ctx()
    q, k, v = qkv.split([Hq * D, Hk * D, Hk * D + 16], 1)
    tl.tl_qk_norm_rope_cache(c, dims, q, row, k, row, v, row, qo, Hq * D, pools[0], pools[1], slots.to(dev()), wq, wk, EPS, pos, cs, MAXPOS, rot, True,
                             torch.cuda.current_stream())
    torch.cuda.synchronize()
    s, p = slots.numpy().astype(np.int64), pos.cpu().numpy()
    keep = (s >= 0) & (s < n_pages * page)
    kc, vc = (torch.as_strided(x, (n_pages, Hk, page, D), (step, page * D, D, 1)) for x in pools)
    at = torch.from_numpy(np.where(keep, s, 0)).to(dev())
    close(qo, q, Hq, wq, p, cs, rot, True, keep)
    close(kc[at // page, :, at % page].reshape(T, Hk * D), k, Hk, wk, p, cs, rot, True, keep)
    kd = torch.from_numpy(keep).to(dev())
    assert torch.equal(vc[at // page, :, at % page].reshape(T, Hk * D)[kd], v[:, :Hk * D][kd])
    assert (qo[~kd] == 7).all()
    used = torch.zeros(n_pages * page, dtype=torch.bool, device=dev())
    used[at[kd]] = True
    for x, pool in zip((kc, vc), pools):
        assert (x.transpose(1, 2).reshape(n_pages * page, Hk, D)[~used] == 7).all()
        if stride:
            assert (pool.view(n_pages, step)[:, Hk * page * D:] == 7).all()
    tl.tl_ctx_destroy(c)


def test_cache_offsets_beyond_32_bits():
    T, Hq, Hk, page, step = 4, 2, 1, 16, 1 << 28
    n_pages = 20
    qkv, (wq, wk), pos = draw(T, Hq, Hk, 6)
    pools = [torch.empty(n_pages * step, dtype=torch.bfloat16, device=dev()) for _ in range(2)]
    slots = ints([17 * 16 + 3, 19 * 16 + 15, 0, 16])
    dims = tl.tl_paged_dims(batch=1, max_tokens=T, max_blocks=n_pages, page_size=page, n_pages=n_pages, heads_q=Hq, heads_kv=Hk, head_dim=D, page_stride=step)
    q, k, v = qkv.split([Hq * D, D, D], 1)
    qo, cs, row = torch.zeros(T, Hq * D, dtype=torch.bfloat16, device=dev()), angles(64), qkv.stride(0)
    c = ctx()
    tl.tl_qk_norm_rope_cache(c, dims, q, row, k, row, v, row, qo, Hq * D, *pools, slots, wq, wk, EPS, pos, cs, MAXPOS, 64, False)
    torch.cuda.synchronize()
    got = [torch.stack([x[s // 16 * step + s % 16 * D:][:D] for s in slots.tolist()]) for x in pools]
    close(got[0], k, 1, wk, pos.cpu().numpy(), cs, 64, False)
    assert torch.equal(got[1], v)
    tl.tl_ctx_destroy(c)
