"""tl_paged_slots against its definition, request by request: whole numbers, equal or wrong."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from oracle import paged as ref
from tests.paged_util import ctx, dev, ints

pytestmark = pytest.mark.gpu
GUARD = -77


def run(cached, new, page=16, T=None, max_new=0, width=None, n_pages=4000, n_free=None, free_from=0, in_place=False, seed=0, stream=None):
    rng = np.random.default_rng(seed)
    B = len(cached)
    T = max(1, sum(max(n, 0) for n in new)) if T is None else T
    width = max(-(-(max(c, 0) + max(n, 0)) // page) for c, n in zip(cached, new)) + 1 if width is None else width
    order = rng.permutation(n_pages)
    table = rng.integers(0, n_pages, (B, width))
    free = order[:n_pages if n_free is None else n_free]
    d = dict(ctx=ints(cached), new=ints(new), free=ints(free) if len(free) else None, frm=ints([free_from]), table=ints(table))
    if in_place:
        seq, to = d["ctx"], d["frm"]
    else:
        seq, to = ints([GUARD] * B), ints([GUARD])
    out = dict(query_start=ints([GUARD] * (B + 3)), slots=ints([GUARD] * (T + 5)), positions=ints([GUARD] * (T + 5)), counts=ints([GUARD] * 6))
    c = ctx()
    dims = tl.tl_paged_dims(batch=B, max_tokens=T, max_new=max_new, max_blocks=width, page_size=page, n_pages=n_pages, heads_q=1, heads_kv=1, head_dim=128)
    tl.tl_paged_slots(c, dims, d["ctx"], d["new"], d["free"], len(free), d["frm"], to, d["table"], out["query_start"], seq, out["slots"], out["positions"],
                      out["counts"], stream)
    torch.cuda.synchronize()
    tl.tl_ctx_destroy(c)
    want = ref.slots(cached, new, free, free_from, table, T, max_new or T, page, n_pages)
    got = {k: v.cpu().numpy() for k, v in out.items()}
    assert np.array_equal(d["table"].cpu().numpy(), want["table"])
    assert np.array_equal(seq.cpu().numpy(), want["seq_lens"]) and int(to[0]) == want["free_to"]
    for k, n in (("query_start", B + 1), ("slots", T), ("positions", T), ("counts", 4)):
        assert np.array_equal(got[k][:n], want[k]), k
        assert (got[k][n:] == GUARD).all(), f"{k}: written behind its end"
    return want


@pytest.mark.parametrize("page", [16, 32, 256])
def test_decode_step(page):
    run([0, 1, page - 1, page, page + 1, 5 * page, 1000], [1] * 7, page=page)


@pytest.mark.parametrize("B", [1, 63, 64, 65, 1000, 1025, 4096])
def test_batches(B):
    rng = np.random.default_rng(B)
    run(list(rng.integers(0, 200, B)), list(rng.integers(0, 6, B)), n_pages=40000, seed=B)


@pytest.mark.parametrize("lens", [[5000], [4096, 1], [1, 9000, 0, 3], [40000]], ids=str)
def test_long_prompts(lens):
    """More than one workgroup's share of tokens."""
    run([7 * i for i in range(len(lens))], lens, n_pages=5000)


def test_padding_rows_and_requests():
    w = run([10, 0, 40, 0], [3, 0, 2, 0], T=64)
    assert (w["slots"][5:] == -1).all()
    run([10, 0], [0, 0], T=8)
    run([100] * 3, [0] * 3, T=6000)


def test_free_list_runs_out():
    w = run([15, 16, 0], [2, 40, 100], n_free=4, free_from=1)
    assert w["counts"][2] > 0 and (w["slots"] == -1).any()
    run([15, 16], [2, 40], n_free=0)
    run([3, 3], [50, 5000], n_free=7, free_from=7)
    run([3, 3], [50, 50], n_free=7, free_from=900)          # more used than there are


def test_tokens_that_do_not_fit():
    run([0, 0, 0], [10, 10, 10], T=17)                      # rows
    run([0, 5, 0], [10, 100, 3], T=200, max_new=40)         # tokens of one request
    run([60, 10, 200], [10, 10, 1], width=4)                # columns of the table
    run([-3, 10], [5, -2])                                  # lengths below zero count as zero
    run([0] * 3, [3000] * 3, T=8000)


@pytest.mark.parametrize("lens", [[1, 1, 1], [100, 100, 100], [3000, 2000, 1]], ids=str)
def test_in_place(lens):
    run([5, 31, 64], lens, in_place=True, free_from=3)


def test_captured_step_feeds_itself():
    """One captured decode step, replayed: lengths and the free list move on in place, tables grow."""
    page, B, T, width, n_pages = 16, 5, 8, 6, 64
    rng = np.random.default_rng(3)
    cached, new = [0, 14, 15, 16, 40], [1, 1, 1, 0, 1]
    free = rng.permutation(n_pages)
    table = np.full((B, width), -5)
    used = 0
    for b, c in enumerate(cached):
        for j in range(-(-c // page)):
            table[b, j] = free[used]
            used += 1
    t = dict(ctx=ints(cached), new=ints(new), free=ints(free), frm=ints([used]), table=ints(table), qs=ints([0] * (B + 1)), slots=ints([0] * T),
             pos=ints([0] * T), counts=ints([0] * 4))
    c = ctx()
    dims = tl.tl_paged_dims(batch=B, max_tokens=T, max_new=1, max_blocks=width, page_size=page, n_pages=n_pages, heads_q=1, heads_kv=1, head_dim=128)

    def step():
        tl.tl_paged_slots(c, dims, t["ctx"], t["new"], t["free"], n_pages, t["frm"], t["frm"], t["table"], t["qs"], t["ctx"], t["slots"], t["pos"], t["counts"],
                          torch.cuda.current_stream())

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        step()
    for _ in range(20):
        want = ref.slots(cached, new, free, used, table, T, 1, page, n_pages)
        g.replay()
        torch.cuda.synchronize()
        cached, used, table = list(want["seq_lens"]), want["free_to"], want["table"]
        for k, x in (("ctx", cached), ("frm", [used]), ("table", table), ("slots", want["slots"]), ("pos", want["positions"]), ("counts", want["counts"])):
            assert np.array_equal(t[k].cpu().numpy(), x), k
    tl.tl_ctx_destroy(c)
