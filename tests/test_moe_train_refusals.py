"""Argument checks of a mixture-of-experts layer's training operators, on the CPU: a host-only context answers the size queries, every wrong
argument is refused with its own status, and a call whose arguments are right is stopped only by the context."""
import pytest

import paper_2503_20313_amd as tl

ARG, SHAPE, SMALL = tl.TL_ERR_INVALID_ARG, tl.TL_ERR_UNSUPPORTED_SHAPE, tl.TL_ERR_WORKSPACE_TOO_SMALL
P = 4096          # stands for a device address: nothing reads it here
BIG = 1 << 40


@pytest.fixture
def ctx():
    c = tl.tl_ctx_create_host(256, world_size=1, rank=0, channels_per_rank=1)
    yield c
    tl.tl_ctx_destroy(c)


def refused(status, text, f, *args):
    with pytest.raises(tl.TileLinkError) as e:
        f(*args)
    assert e.value.status == status and text in str(e.value), str(e.value)


def _call(f, **base):
    def make(**kw):
        assert not set(kw) - set(base), kw
        a = dict(base, **kw)
        return lambda c: f(c, *a.values())
    make.base = base
    return make


ROWS = dict(row_pos=P, T=9, H=64, topk=3, max_rows=20)
PRODUCT = dict(expert_offsets=P, max_rows=50, K=64, N=96, E=4)
WS = dict(workspace=P, ws_bytes=BIG)
CALLS = dict(
    sort=_call(tl.tl_moe_sort, topk_ids=P, T=9, topk=3, first_expert=0, E=8, expert_offsets=P, sorted_row=P, row_pos=P, **WS),
    dispatch=_call(tl.tl_moe_dispatch, x=P, **ROWS, xs=P),
    dispatch_grad=_call(tl.tl_moe_dispatch_grad, dxs=P, **ROWS, dx=P),
    combine=_call(tl.tl_moe_combine, ys=P, topk_w=P, **ROWS, add=P, out=P),
    combine_grad=_call(tl.tl_moe_combine_grad, dout=P, ys=P, topk_w=P, **ROWS, dys=P, dtopk_w=P),
    route_grad=_call(tl.tl_moe_route_grad, gate_logits=P, topk_ids=P, dtopk_w=P, T=9, E=8, topk=3, renormalize=1, dlogits=P),
    gemm=_call(tl.tl_moe_gemm, x=P, w=P, **PRODUCT, y=P, **WS),
    grad_x=_call(tl.tl_moe_gemm_grad_x, dy=P, w=P, **PRODUCT, dx=P, **WS),
    grad_w=_call(tl.tl_moe_gemm_grad_w, x=P, dy=P, **PRODUCT, dw_add=P, dw=P, dw_f32=1, **WS))
WAYS = dict(gemm=tl.TL_MOE_FORWARD, grad_x=tl.TL_MOE_GRAD_X, grad_w=tl.TL_MOE_GRAD_W)


@pytest.mark.parametrize("name", list(CALLS))
def test_a_right_call_needs_a_real_context(ctx, name):
    refused(ARG, "tl_ctx_create_host", CALLS[name](), ctx)
    refused(ARG, "context is null", CALLS[name](), None)


POINTERS = [(n, k) for n, f in CALLS.items() for k, v in f.base.items() if v == P]


@pytest.mark.parametrize("name,arg", POINTERS, ids=str)
def test_null_and_misaligned_pointers(ctx, name, arg):
    if arg in ("add", "dw_add"):
        refused(ARG, "tl_ctx_create_host", CALLS[name](**{arg: None}), ctx)
    else:
        refused(ARG, "null", CALLS[name](**{arg: None}), ctx)
    refused(ARG, "aligned", CALLS[name](**{arg: P + 2}), ctx)


SIZES = [(n, k) for n, f in CALLS.items() for k in ("T", "H", "topk", "max_rows", "K", "N", "E") if k in f.base]


@pytest.mark.parametrize("name,arg", SIZES, ids=str)
def test_sizes_are_positive(ctx, name, arg):
    for v in (0, -1, -(1 << 31)):
        refused(ARG, "positive", CALLS[name](**{arg: v}), ctx)


@pytest.mark.parametrize("name,status,text,change", [
    ("sort", ARG, "first_expert", dict(first_expert=-1)), ("sort", ARG, "first_expert", dict(first_expert=(1 << 31) - 7)), ("sort", SHAPE, "256", dict(E=257)), ("sort", SHAPE, "32", dict(topk=33)),
    ("sort", SHAPE, "2^20", dict(T=(1 << 20) // 3 + 1)), ("sort", SHAPE, "31 bits", dict(T=1 << 30)),
    ("route_grad", SHAPE, "256", dict(E=257)), ("route_grad", SHAPE, "topk <= E", dict(topk=9)), ("route_grad", SHAPE, "2^24", dict(T=(1 << 24) + 1)),
    ("grad_w", ARG, "fp32", dict(dw_f32=0)),
] + [(n, SHAPE, "multiple of 8", dict(H=68)) for n in ("dispatch", "dispatch_grad", "combine", "combine_grad")]
  + [(n, SHAPE, "more than 32", dict(topk=33)) for n in ("dispatch", "dispatch_grad", "combine", "combine_grad")]
  + [(n, SHAPE, "31 bits", dict(T=1 << 30)) for n in ("dispatch", "dispatch_grad", "combine", "combine_grad")]
  + [(n, SHAPE, "multiples of 8", d) for n in WAYS for d in (dict(K=60), dict(N=90))]
  + [(n, SHAPE, "256", dict(E=257)) for n in WAYS] + [(n, SHAPE, "2^20", d) for n in WAYS for d in (dict(K=(1 << 20) + 8), dict(N=(1 << 20) + 8))]
  + [("grad_w", SHAPE, "2^22", dict(K=1 << 20, N=1 << 16))] + [(n, ARG, "128-byte", dict(workspace=P + 64)) for n in WAYS], ids=str)
def test_values(ctx, name, status, text, change):
    refused(status, text, CALLS[name](**change), ctx)


def test_workspaces(ctx):
    """What the queries ask for is what the calls accept."""
    for kw in (dict(T=1, topk=1, E=1), dict(T=341, topk=3, E=8), dict(T=342, topk=3, E=256), dict(T=1 << 17, topk=8, E=256)):
        n = tl.tl_moe_sort_query(ctx, **kw)
        refused(ARG, "tl_ctx_create_host", CALLS["sort"](**kw, ws_bytes=n), ctx)
        refused(SMALL, "needed", CALLS["sort"](**kw, ws_bytes=n - 1), ctx)
    for name, way in WAYS.items():
        for kw in (dict(max_rows=1, K=8, N=8, E=1), dict(max_rows=320, K=2048, N=1536, E=32), dict(max_rows=65536, K=512, N=512, E=1),
                   dict(max_rows=16384, K=4096, N=1792, E=256)):
            n = tl.tl_moe_gemm_query(ctx, way, **kw)
            assert n % 128 == 0 and n > 0
            refused(ARG, "tl_ctx_create_host", CALLS[name](**kw, ws_bytes=n), ctx)
            refused(SMALL, "needed", CALLS[name](**kw, ws_bytes=n - 1), ctx)
    refused(ARG, "three products", tl.tl_moe_gemm_query, ctx, 3, 8, 8, 8, 1)
    refused(ARG, "context is null", tl.tl_moe_gemm_query, None, 0, 8, 8, 8, 1)
    refused(ARG, "context is null", tl.tl_moe_sort_query, None, 8, 1, 1)


def test_right_calls_at_the_limits(ctx):
    refused(ARG, "tl_ctx_create_host", CALLS["sort"](T=1 << 15, topk=32, E=256), ctx)
    refused(ARG, "tl_ctx_create_host", CALLS["sort"](first_expert=(1 << 31) - 8, E=8), ctx)
    refused(ARG, "tl_ctx_create_host", CALLS["route_grad"](T=1 << 24, E=256, topk=32), ctx)
    refused(ARG, "tl_ctx_create_host", CALLS["dispatch"](T=(1 << 26) - 1, topk=32, H=8, max_rows=(1 << 31) - 1), ctx)
    refused(ARG, "tl_ctx_create_host", CALLS["grad_w"](dw_add=None, dw_f32=0), ctx)
    refused(ARG, "tl_ctx_create_host", CALLS["gemm"](max_rows=(1 << 31) - 1, K=1 << 20, N=8, E=256), ctx)
