"""Argument checks of the paged-cache operators, on the CPU: a host-only context answers the size queries, every wrong argument is
refused with its own status, and a call whose arguments are right is stopped only by the context."""
import pytest

import paper_2503_20313_amd as tl

ARG, SHAPE, SMALL = tl.TL_ERR_INVALID_ARG, tl.TL_ERR_UNSUPPORTED_SHAPE, tl.TL_ERR_WORKSPACE_TOO_SMALL
P = 4096          # stands for a device address: nothing reads it here


@pytest.fixture
def ctx():
    c = tl.tl_ctx_create_host(256, world_size=1, rank=0, channels_per_rank=1)
    yield c
    tl.tl_ctx_destroy(c)


def dims(**kw):
    base = dict(batch=4, max_tokens=64, max_new=32, max_blocks=10, page_size=16, n_pages=50, heads_q=8, heads_kv=2, head_dim=128, window=0, page_stride=0)
    base.update(kw)
    return tl.tl_paged_dims(**base)


def refused(status, text, f, *args):
    with pytest.raises(tl.TileLinkError) as e:
        f(*args)
    assert e.value.status == status and text in str(e.value), str(e.value)


BAD_DIMS = [(ARG, "positive", dict(batch=0)), (ARG, "positive", dict(max_tokens=-1)), (ARG, "positive", dict(max_blocks=0)), (ARG, "positive", dict(n_pages=0)),
            (ARG, "positive", dict(heads_q=0)), (ARG, "positive", dict(heads_kv=-2)), (ARG, "max_new", dict(max_new=65)), (ARG, "max_new", dict(max_new=-1)),
            (ARG, "window", dict(window=-1)), (SHAPE, "4096", dict(batch=4097)), (SHAPE, "262144", dict(max_tokens=(1 << 18) + 1)),
            (SHAPE, "head_dim", dict(head_dim=64)), (SHAPE, "page_size", dict(page_size=8)), (SHAPE, "page_size", dict(page_size=48)),
            (SHAPE, "page_size", dict(page_size=512)), (SHAPE, "divide", dict(heads_q=7)), (SHAPE, "1024", dict(heads_q=2048)),
            (SHAPE, "32 bits", dict(n_pages=1 << 27)), (SHAPE, "2^28", dict(max_blocks=(1 << 24) + 1)), (ARG, "page_stride", dict(page_stride=4095)),
            (ARG, "page_stride", dict(page_stride=-8)), (SHAPE, "multiple of 8", dict(page_stride=4100))]


@pytest.mark.parametrize("status,text,change", BAD_DIMS, ids=lambda x: str(x) if isinstance(x, dict) else "")
def test_dims(ctx, status, text, change):
    refused(status, text, tl.tl_paged_query, ctx, dims(**change))
    refused(status, text, slots_call(dims=dims(**change)), ctx)
    refused(status, text, schedule_call(dims=dims(**change)), ctx)
    refused(status, text, attention_call(dims=dims(**change)), ctx)
    refused(status, text, cache_call(dims=dims(**change)), ctx)


def _call(f, base):
    def make(**kw):
        assert not set(kw) - set(base), kw
        a = dict(base, **kw)
        return lambda c: f(c, *a.values())
    make.base = base
    return make


slots_call = _call(tl.tl_paged_slots, dict(dims=dims(), ctx_lens=P, new_lens=P, free_pages=P, n_free=9, free_from=P, free_to=P, block_table=P, query_start=P,
                                           seq_lens=P, slots=P, positions=P, counts=P))
schedule_call = _call(tl.tl_paged_schedule, dict(dims=dims(), query_start=P, seq_lens=P, schedule=P, schedule_bytes=1 << 20))
attention_call = _call(tl.tl_paged_attention, dict(dims=dims(), q=P, q_stride=1024, k_cache=P, v_cache=P, block_table=P, schedule=P, o=P, o_stride=1024, lse=P,
                                                   scale=0.1, workspace=P, ws_bytes=1 << 40))
rope_call = _call(tl.tl_qk_norm_rope, dict(q=P, q_stride=1024, k=P, k_stride=256, q_out=P, q_out_stride=1024, k_out=P, k_out_stride=256, T=5, heads_q=8, heads_kv=2,
                                           head_dim=128, q_weight=P, k_weight=P, eps=1e-6, positions=P, cos_sin=P, max_position=10, rot_dim=128, interleaved=0))
cache_call = _call(tl.tl_qk_norm_rope_cache, dict(dims=dims(), q=P, q_stride=1024, k=P, k_stride=256, v=P, v_stride=256, q_out=P, q_out_stride=1024, k_cache=P,
                                                  v_cache=P, slots=P, q_weight=P, k_weight=P, eps=1e-6, positions=P, cos_sin=P, max_position=10, rot_dim=128,
                                                  interleaved=0))
CALLS = dict(slots=slots_call, schedule=schedule_call, attention=attention_call, rope=rope_call, cache=cache_call)


@pytest.mark.parametrize("name", list(CALLS))
def test_a_right_call_needs_a_real_context(ctx, name):
    refused(ARG, "tl_ctx_create_host", CALLS[name](), ctx)
    refused(ARG, "context is null", CALLS[name](), None)
    if name != "rope":
        refused(ARG, "dims", CALLS[name](dims=None), ctx)


OPTIONAL = dict(slots={"free_from", "free_to"}, attention={"lse"}, rope=set(), cache=set(), schedule=set())
POINTERS = [(n, k) for n, f in CALLS.items() for k, v in f.base.items() if v == P]


@pytest.mark.parametrize("name,arg", POINTERS, ids=str)
def test_null_and_misaligned_pointers(ctx, name, arg):
    if arg in OPTIONAL[name]:
        refused(ARG, "tl_ctx_create_host", CALLS[name](**{arg: None}), ctx)
    else:
        refused(ARG, "together" if "weight" in arg else "rotation" if name != "slots" and arg in ("positions", "cos_sin") else "null", CALLS[name](**{arg: None}), ctx)
    refused(ARG, "aligned", CALLS[name](**{arg: P + 2}), ctx)


@pytest.mark.parametrize("name,status,text,change", [
    ("slots", ARG, "n_free", dict(n_free=-1)),
    ("schedule", SMALL, "needed", dict(schedule_bytes=64)),
    ("attention", SMALL, "needed", dict(ws_bytes=256)),
    ("attention", ARG, "128-byte", dict(workspace=P + 64)), ("attention", ARG, "scale", dict(scale=0.0)), ("attention", ARG, "scale", dict(scale=float("nan"))), ("attention", ARG, "scale", dict(scale=float("inf"))),
    ("attention", ARG, "stride", dict(q_stride=1023)), ("attention", SHAPE, "multiples of 8", dict(o_stride=1028)),
    ("rope", ARG, "positive", dict(T=0)), ("rope", SHAPE, "head_dim", dict(head_dim=64)), ("rope", SHAPE, "rot_dim", dict(rot_dim=24)),
    ("rope", SHAPE, "rot_dim", dict(rot_dim=144)), ("rope", ARG, "eps", dict(eps=-1.0)), ("rope", ARG, "eps", dict(eps=float("nan"))),
    ("rope", ARG, "rotation", dict(max_position=0)), ("rope", ARG, "stride", dict(q_stride=896)), ("rope", ARG, "stride", dict(k_out_stride=0)),
    ("rope", SHAPE, "multiples of 8", dict(k_stride=260)), ("rope", SHAPE, "multiples of 8", dict(k_out_stride=260)), ("rope", SHAPE, "1024", dict(heads_kv=1025)),
    ("cache", ARG, "stride", dict(v_stride=128)), ("cache", SHAPE, "multiples of 8", dict(v_stride=260)), ("cache", ARG, "stride", dict(q_out_stride=8)),
], ids=str)
def test_values(ctx, name, status, text, change):
    refused(status, text, CALLS[name](**change), ctx)


def test_no_rotation_and_no_norm_are_right_calls(ctx):
    refused(ARG, "tl_ctx_create_host", rope_call(rot_dim=0, positions=None, cos_sin=None, max_position=0), ctx)
    refused(ARG, "tl_ctx_create_host", cache_call(q_weight=None, k_weight=None), ctx)
    refused(ARG, "tl_ctx_create_host", slots_call(free_pages=None, n_free=0), ctx)


def test_in_place_has_one_stride(ctx):
    """Another stride in place would write rows over rows that are still to be read; a single row has none."""
    for call in (rope_call, cache_call):
        refused(ARG, "in place", call(q_stride=2048), ctx)
        refused(ARG, "in place", call(q_out_stride=1032), ctx)
        refused(ARG, "tl_ctx_create_host", call(q_stride=2048, q_out_stride=2048), ctx)
        refused(ARG, "tl_ctx_create_host", call(q_stride=2048, q_out=2 * P), ctx)
    refused(ARG, "in place", rope_call(k_out_stride=512), ctx)
    refused(ARG, "tl_ctx_create_host", rope_call(q_stride=2048, k_stride=512, T=1), ctx)


def test_sizes(ctx):
    """What the query asks for is what the calls accept, and grows with the batch; a decode step needs no room for tiles."""
    for kw in (dict(), dict(max_new=1), dict(heads_q=64, heads_kv=1), dict(batch=4096, max_tokens=1 << 18, max_new=0), dict(heads_q=1024, heads_kv=1024),
               dict(max_blocks=1 << 24, n_pages=(1 << 27) - 1)):
        z = tl.tl_paged_query(ctx, dims(**kw))
        assert z["schedule_bytes"] % 16 == 0 and z["ws_bytes"] % 16 == 0
        refused(ARG, "tl_ctx_create_host", schedule_call(dims=dims(**kw), schedule_bytes=z["schedule_bytes"]), ctx)
        refused(SMALL, "needed", schedule_call(dims=dims(**kw), schedule_bytes=z["schedule_bytes"] - 1), ctx)
        refused(ARG, "tl_ctx_create_host", attention_call(dims=dims(**kw), q_stride=1 << 20, o_stride=1 << 20, ws_bytes=z["ws_bytes"]), ctx)
        refused(SMALL, "needed", attention_call(dims=dims(**kw), q_stride=1 << 20, o_stride=1 << 20, ws_bytes=z["ws_bytes"] - 1), ctx)
    one = tl.tl_paged_query(ctx, dims(max_new=1))
    assert one["tile_items"] == 0 and one["few_items"] >= 4
    assert tl.tl_paged_query(ctx, dims(heads_q=66, heads_kv=1))["few_items"] == 0
