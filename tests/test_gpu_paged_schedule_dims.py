"""tl_paged_attention with a schedule that was made for other dims: no work is found in it, nothing is written."""
import pytest
import torch

import paper_2503_20313_amd as tl
from tests.paged_util import D, SCALE, ctx, dev, ints

pytestmark = pytest.mark.gpu
GUARD = -7


def paged_dims(batch, max_tokens, max_new, max_blocks, page_stride=0):
    return tl.tl_paged_dims(batch=batch, max_tokens=max_tokens, max_new=max_new, max_blocks=max_blocks, page_size=16, n_pages=8192, heads_q=32, heads_kv=8,
                            head_dim=D, page_stride=page_stride)


def made_schedule(c, dims, new, seq, behind=0):
    """A schedule for `dims` of the first requests given, and `behind` words after it."""
    z = tl.tl_paged_query(c, dims)
    n = z["schedule_bytes"] // 4
    out = torch.full((n + behind,), GUARD, dtype=torch.int32, device=dev())
    new, seq = (list(x) + [0] * (dims.batch - len(x)) for x in (new, seq))
    start = torch.tensor([0] + new).cumsum(0)
    tl.tl_paged_schedule(c, dims, ints(start), ints(seq), out[:n], z["schedule_bytes"], torch.cuda.current_stream())
    return out


def attend(c, dims, schedule):
    """One call under `dims`; returns whether anything was written."""
    T, H = dims.max_tokens, dims.heads_q
    z = tl.tl_paged_query(c, dims)
    cache = torch.zeros(dims.n_pages * dims.heads_kv * 16 * D, dtype=torch.bfloat16, device=dev())
    q = torch.randn(T, H * D, device=dev()).to(torch.bfloat16)
    o, lse = torch.full((T, H * D), 7.0, dtype=torch.bfloat16, device=dev()), torch.full((T, H), 7.0, device=dev())
    table = torch.zeros(dims.batch, dims.max_blocks, dtype=torch.int32, device=dev())
    ws = torch.zeros(z["ws_bytes"] // 4, device=dev())
    tl.tl_paged_attention(c, dims, q, H * D, cache, cache, table, schedule, o, H * D, lse, SCALE, ws, z["ws_bytes"], torch.cuda.current_stream())
    torch.cuda.synchronize()
    return bool((o != 7).any() or (lse != 7).any() or ws.any())


def test_dims_that_hash_alike():
    """Two ordinary dims that a multiplicative hash of their fields does not tell apart, each under the other's schedule."""
    one, two = paged_dims(128, 1024, 13, 64), paged_dims(256, 4096, 2988, 2048)
    c = ctx()
    s1, s2 = made_schedule(c, one, [1, 13], [1000, 13]), made_schedule(c, two, [1, 2988], [30000, 2988])
    torch.cuda.synchronize()
    assert int(s1[1]) > 0 and int(s2[1]) > 0
    assert not attend(c, one, s2)
    assert attend(c, one, s1)
    tl.tl_ctx_destroy(c)


@pytest.mark.parametrize("max_new", [1, 512])
def test_a_schedule_of_smaller_dims_that_ends_early(max_new):
    """The buffer of one request's schedule, under the dims of a large batch.  What lies behind its end looks like items."""
    c = ctx()
    small, large = paged_dims(1, 1, 1, 64), paged_dims(4096, 8192, max_new, 64)
    z = tl.tl_paged_query(c, large)
    s = made_schedule(c, small, [1], [100], behind=z["schedule_bytes"] // 4)
    s[tl.tl_paged_query(c, small)["schedule_bytes"] // 4:] = 1
    assert not attend(c, large, s)
    tl.tl_ctx_destroy(c)


def test_one_schedule_for_layers_whose_pages_lie_differently():
    c = ctx()
    s = made_schedule(c, paged_dims(128, 1024, 13, 64), [1], [20])
    dims = paged_dims(128, 1024, 13, 64, page_stride=16 * 8 * D + 64)
    z = tl.tl_paged_query(c, dims)
    cache = torch.ones(dims.n_pages * dims.page_stride, dtype=torch.bfloat16, device=dev())
    q, o = torch.zeros(1024, 32 * D, dtype=torch.bfloat16, device=dev()), torch.zeros(1024, 32 * D, dtype=torch.bfloat16, device=dev())
    ws = torch.zeros(z["ws_bytes"] // 4, device=dev())
    tl.tl_paged_attention(c, dims, q, 32 * D, cache, cache, torch.zeros(128, 64, dtype=torch.int32, device=dev()), s, o, 32 * D, None, SCALE, ws, z["ws_bytes"],
                          torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert (o[0] == 1).all() and (o[1:] == 0).all()
    tl.tl_ctx_destroy(c)
