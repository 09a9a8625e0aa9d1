"""Sizes whose launch would have 2^32 work items or more, of which the runtime silently leaves the last out: refused, on the CPU."""
import pytest

import paper_2503_20313_amd as tl
from tests.test_paged_refusals import ARG, SHAPE, attention_call, cache_call, ctx, dims, refused, rope_call, schedule_call  # noqa: F401 (ctx is a fixture)


def workgroups(z, heads_kv):
    return (z["few_items"] + z["tile_items"]) * heads_kv


def test_tiles_of_the_largest_steps(ctx):  # noqa: F811
    """4096 requests over 2^18 rows: at 1024 key heads 1.125 * 2^32 threads, of which an eighth of 2^32 was started."""
    most = dict(batch=4096, max_tokens=1 << 18, max_new=0)
    bad = dims(heads_q=1024, heads_kv=1024, **most)
    refused(SHAPE, "one launch", tl.tl_paged_query, ctx, bad)
    refused(SHAPE, "one launch", schedule_call(dims=bad), ctx)
    refused(SHAPE, "one launch", attention_call(dims=bad, q_stride=1 << 20, o_stride=1 << 20), ctx)
    refused(SHAPE, "one launch", cache_call(dims=bad), ctx)
    last = 0
    for heads in range(1, 1025):
        try:
            z = tl.tl_paged_query(ctx, dims(heads_q=heads, heads_kv=heads, **most))
        except tl.TileLinkError:
            break
        last = heads
        assert workgroups(z, heads) * 512 < 1 << 32
    assert (workgroups(z, last) + workgroups(z, last) // last) * 512 >= 1 << 32, "the next one would have fitted"


@pytest.mark.parametrize("name", ["rope", "cache"])
def test_rows_and_heads(ctx, name):  # noqa: F811
    if name == "rope":
        kw = dict(heads_q=32, heads_kv=8, q_stride=4096, k_stride=1024, q_out_stride=4096, k_out_stride=1024)
        rows = (2 ** 24 - 1) * 16 // 20          # 20 pairs of heads a row, 16 a workgroup of 256 threads
        refused(ARG, "tl_ctx_create_host", rope_call(T=rows, **kw), ctx)
        refused(SHAPE, "one launch", rope_call(T=rows + 1, **kw), ctx)
        refused(SHAPE, "one launch", rope_call(T=2 ** 31 - 1, **kw), ctx)
    else:
        row = dict(q_stride=1 << 17, k_stride=1 << 17, v_stride=1 << 17, q_out_stride=1 << 17)
        few = dict(batch=1, max_new=1, heads_q=1024, heads_kv=1024)
        refused(ARG, "tl_ctx_create_host", cache_call(dims=dims(max_tokens=(2 ** 24 - 1) * 16 // 1536, **few), **row), ctx)
        refused(SHAPE, "one launch", cache_call(dims=dims(max_tokens=1 << 18, **few), **row), ctx)
