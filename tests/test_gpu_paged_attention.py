"""tl_paged_schedule + tl_paged_attention against the plain definition in 64 bits: lengths, head layouts, pages, windows, strides,
missing pages, values that must not matter, long offsets, graphs and streams."""
import math

import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from tests.paged_util import D, Batch, check_attention, ctx, dev, ints, np64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [(1, 1), (2, 1), (4, 2), (5, 1), (8, 8), (16, 2), (16, 1), (32, 1)], ids=str)
@pytest.mark.parametrize("page", [16, 64])
def test_single_tokens(heads, page):
    """One new token per request; contexts around the unit of 32 keys, the block of 64 and the page."""
    cached = [0, 1, 14, 15, 16, 30, 31, 32, 33, 62, 63, 64, 65, 127, 128, 300]
    b = Batch(cached, [1] * len(cached), *heads, page=page, seed=1)
    b.run()
    check_attention(b)


@pytest.mark.parametrize("cached", [0, 1, 17, 63, 64, 200])
@pytest.mark.parametrize("new", [2, 5, 31, 33, 64, 65, 130])
@pytest.mark.parametrize("heads", [(2, 2), (6, 2)], ids=str)
def test_one_chunk(cached, new, heads):
    b = Batch([cached], [new], *heads, page=16, seed=2)
    b.run()
    check_attention(b)


@pytest.mark.parametrize("heads", [(2, 1), (7, 1), (40, 1), (12, 4)], ids=str)
@pytest.mark.parametrize("window", [0, 1, 16, 100])
def test_mixed_batch(heads, window):
    """Single tokens, chunks, requests without new tokens, in one call; 40 heads to a key head are too many for the few-row kernel."""
    b = Batch([40, 0, 7, 129, 64, 500, 3], [1, 33, 0, 1, 70, 3, 2], *heads, page=32, window=window, seed=3)
    b.run()
    check_attention(b)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_page_sizes(page):
    b = Batch([255, 256, 257, 20], [1, 40, 3, 1], 4, 2, page=page, seed=4)
    b.run()
    check_attention(b)


@pytest.mark.parametrize("heads,cached,new", [((4, 1), [6000], [1]), ((16, 1), [9000], [1]), ((2, 1), [20000, 300], [1, 3]), ((8, 8), [3000, 10], [1, 1]), ((2, 1), [5000], [40]), ((1, 1), [2500, 0], [300, 1])], ids=str)
def test_cut_key_axis(heads, cached, new):
    """Few rows and long contexts: the key axis is cut, the runs are joined."""
    b = Batch(cached, new, *heads, page=16, seed=5)
    z = b.buffers(c := ctx())
    b.schedule_call(c)
    torch.cuda.synchronize()
    hdr = b.schedule[:3].tolist()
    tl.tl_ctx_destroy(c)
    assert hdr[1] > len(cached), "this case is meant to cut the key axis"
    assert hdr[1] <= z["few_items"] + z["tile_items"]
    b.run()
    check_attention(b)


@pytest.mark.parametrize("new", [1, 3, 60])
def test_cut_key_axis_in_a_window(new):
    b = Batch([9000, 100], [new, 1], 4, 1, page=16, window=5000, seed=19)
    b.run()
    check_attention(b)


def test_largest_batch():
    """4096 requests, the most there can be, of one token each."""
    rng = np.random.default_rng(20)
    b = Batch([int(x) for x in rng.integers(0, 40, 4096)], [1] * 4096, 2, 1, page=16, seed=20)
    b.run()
    check_attention(b)


def test_many_heads():
    b = Batch([70, 5, 200], [1, 2, 40], 384, 128, page=16, seed=21)
    b.run()
    check_attention(b)


def test_very_long_request():
    """300000 keys: runs of hundreds of blocks, tables of thousands of pages, pages looked up again and again."""
    b = Batch([300000], [2], 2, 1, page=16, seed=22)
    b.run()
    check_attention(b)


def test_tokens_without_any_key():
    """More new tokens than the sequence has: the first ones have no position and see nothing."""
    b = Batch([0, 0, 0], [3, 40, 1], 4, 2, seq_lens=[1, 17, 0], seed=6)
    b.run()
    check_attention(b)
    assert (b.o[:2, :4 * D] == 0).all() and torch.isinf(b.lse[:2]).all()


@pytest.mark.parametrize("new", [[1, 1], [50, 3]], ids=str)
def test_missing_pages(new):
    """Entries of the table that are no page: their keys are not attended to; a request with none at all gets zeros."""
    b = Batch([100, 70], new, 8, 2, page=16, seed=7)
    b.table[0, 1] = -1
    b.table[0, 3] = b.n_pages
    b.table[1, :] = -(1 << 31)
    b.run()
    check_attention(b)
    assert (b.o[new[0]:new[0] + new[1], :8 * D] == 0).all()


@pytest.mark.parametrize("heads,max_new", [((4, 2), 1), ((4, 2), 60), ((40, 1), 1)], ids=str)
def test_nothing_new(heads, max_new):
    """A step in which no request has a new token: no item, no row written."""
    b = Batch([50, 0, 3000], [0, 0, 0], *heads, max_new=max_new, spare_rows=60, seed=32)
    b.run()
    assert b.schedule[1:3].tolist() == [0, 0]
    check_attention(b)


@pytest.mark.parametrize("window", [0, 90])
def test_pages_in_several_places(window):
    """Requests with a common beginning list the same pages, and one page stands twice in a table: tables are only read."""
    b = Batch([160, 160, 160, 96], [1, 40, 3, 40], 8, 2, page=32, window=window, seed=31)
    b.table[1, :5] = b.table[2, :5] = b.table[0, :5]
    b.table[3, 2] = b.table[3, 1]
    b.run()
    check_attention(b)


def test_strides():
    """Pages that lie apart, as where the caches of several layers share a buffer."""
    b = Batch([90, 31], [20, 1], 4, 2, page=32, page_stride=2 * 32 * D * 3 + 64, seed=8)
    b.run()
    check_attention(b)


@pytest.mark.parametrize("new", [[1, 1], [90, 1]], ids=str)
def test_offsets_beyond_32_bits(new):
    """A cache of which most elements lie behind 2^32."""
    b = Batch([200, 600], new, 2, 1, page=64, page_stride=1 << 28, spare_pages=12, seed=9)
    assert (b.n_pages - 1) * b.page_stride > 1 << 32
    b.run()
    check_attention(b)


@pytest.mark.parametrize("kind", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("heads", [(2, 1), (16, 1)], ids=str)
@pytest.mark.parametrize("window", [0, 20])
def test_values_of_unseen_keys_do_not_matter(kind, heads, window):
    """Infinities and NaN in keys and values of later tokens and of tokens before the window reach only the rows that see them."""
    b = Batch([30, 5, 64], [4, 100, 2], *heads, page=16, window=window, seed=10)
    for r, at in ((0, 32), (1, 60), (1, 61), (1, 104), (2, 65), (2, 3)):
        b.v[int(b.table[r, at // 16]), :, at % 16, 5] = kind
        b.v[int(b.table[r, at // 16]), :, at % 16, 100] = kind
    b.run()
    check_attention(b)
    b.k[int(b.table[1, 90 // 16]), :, 90 % 16, 7] = kind
    want = b.reference()
    b.run()
    o = np64(b.o[:b.rows, :b.Hq * D]).reshape(b.rows, b.Hq, D)
    assert np.array_equal(np.isfinite(o), np.isfinite(want[0][:b.rows])) and np.array_equal(np.isnan(o), np.isnan(want[0][:b.rows]))


def test_large_scores():
    """Scores in the thousands, of one sign: the running maximum carries them."""
    b = Batch([100, 10], [70, 1], 2, 1, seed=11, q_std=1.0)
    b.qkv[:b.rows] *= 256
    b.k.mul_(16)
    want = b.reference()
    b.run()
    o = np64(b.o[:b.rows, :b.Hq * D]).reshape(b.rows, b.Hq, D)
    # a score's fp32 error is 130 * 2^-24 of its terms' sizes (7 * 4096): 0.22 at most, the weights' ratio is off by exp(2 * 0.22)
    # at most, which moves a weighted mean by that share of the values' spread
    v = np.abs(np64(torch.nan_to_num(b.v.float(), nan=0.0))).max()
    assert np.abs(o - want[0][:b.rows]).max() <= 0.56 * 2 * v and np.isfinite(o).all()
    assert np.median(np.abs(o - want[0][:b.rows])) < 0.01
    assert (np.abs(np64(b.lse[:b.rows]) - want[1][:b.rows]) <= 0.25 + 2.0 ** -20 * np.abs(want[1][:b.rows])).all()


def test_same_bits_again_and_lse_is_optional():
    b = Batch([3000, 40, 1000], [1, 100, 1], 8, 2, page=16, seed=12)
    o, lse = (x.clone() for x in b.run())
    o2, lse2 = b.run()
    assert torch.equal(o.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse, lse2)
    o3, lse3 = b.run(lse=False)
    assert torch.equal(o.view(torch.int16), o3.view(torch.int16)) and (lse3 == 7).all()


def test_many_runs_again_and_again():
    """Long key axes in so many runs that groups of them are joined first, other queries every time, nothing cleared in between: the
    joined parts are this call's."""
    b = Batch([20000, 15000, 900], [1, 1, 1], 4, 1, page=64, seed=18)
    c = ctx()
    b.buffers(c)
    b.schedule_call(c)
    torch.cuda.synchronize()
    assert int(b.schedule[1]) > 34
    for i in range(12):
        b.qkv[:b.rows] = torch.randn(b.rows, b.q_stride, generator=b.g, device=dev()).to(torch.bfloat16)
        want = b.reference() if i in (0, 5, 11) else None
        got = []
        for _ in range(8):
            b.o.fill_(7)
            b.attention_call(c)
            got.append(b.o.clone())
        torch.cuda.synchronize()
        assert all(torch.equal(x.view(torch.int16), got[0].view(torch.int16)) for x in got)
        if want is not None:
            check_attention(b, want)
    tl.tl_ctx_destroy(c)


def test_a_schedule_of_other_dims_is_not_used():
    b = Batch([100, 3], [2, 1], 4, 2, seed=13)
    c = ctx()
    b.buffers(c)
    b.schedule_call(c)
    b.dims.window = 50
    b.attention_call(c)
    torch.cuda.synchronize()
    assert (b.o == 7).all() and (b.lse == 7).all()
    b.schedule.zero_()              # one that was never made
    b.attention_call(c)
    torch.cuda.synchronize()
    assert (b.o == 7).all()
    tl.tl_ctx_destroy(c)


@pytest.mark.parametrize("what", ["below zero", "beyond the rows", "not ascending", "more than max_new", "seq below zero", "seq beyond the table"])
def test_lengths_that_make_no_sense_make_an_empty_table(what):
    b = Batch([100, 3, 50], [2, 1, 40], 4, 2, seed=14)
    c = ctx()
    b.buffers(c)
    guard = torch.full((b.schedule.numel() + 4096,), -1, dtype=torch.int32, device=dev())
    b.schedule = guard[:b.schedule.numel()]
    change = {"below zero": (b.start_d, 0, -1), "beyond the rows": (b.start_d, 3, b.T + 1), "not ascending": (b.start_d, 1, 10), "more than max_new": (b.start_d, 2, 2),
              "seq below zero": (b.seq_d, 2, -1), "seq beyond the table": (b.seq_d, 0, b.width * b.page + 1)}[what]
    change[0][change[1]] = change[2]
    b.schedule_call(c)
    b.attention_call(c)
    torch.cuda.synchronize()
    assert (guard[16:] == -1).all() and int(guard[1]) == 0
    assert (b.o == 7).all() and (b.lse == 7).all()
    tl.tl_ctx_destroy(c)


@pytest.mark.parametrize("B,n", [(1000, 1), (3, 5000), (300, 20)])
def test_schedules_of_every_size(B, n):
    """Every tile's keys are covered once, runs of a tile in order and of one tile together, longest items first, inside the room."""
    rng = np.random.default_rng(B)
    new = [int(x) for x in rng.integers(1, n + 1, B)]
    seq = [int(x) + m for x, m in zip(rng.integers(0, 9000, B), new)]
    start = np.concatenate([[0], np.cumsum(new)])
    c = ctx()
    G, page, width = 4, 64, 256
    d = tl.tl_paged_dims(batch=B, max_tokens=int(start[-1]), max_new=max(new), max_blocks=width, page_size=page, n_pages=1000, heads_q=4 * G, heads_kv=4, head_dim=D)
    z = tl.tl_paged_query(c, d)
    out = torch.full((z["schedule_bytes"] // 4 + 64,), -1, dtype=torch.int32, device=dev())
    tl.tl_paged_schedule(c, d, ints(start), ints(seq), out, z["schedule_bytes"])
    torch.cuda.synchronize()
    tl.tl_ctx_destroy(c)
    out = out.cpu().numpy()
    assert (out[z["schedule_bytes"] // 4:] == -1).all()
    items, cuts = out[1], out[2]
    assert 0 < items <= z["few_items"] + z["tile_items"]
    first = 16 + -(-z["side_by_side"] // 4) * 4
    rec = out[first:first + 12 * items].reshape(items, 12)
    seen, lengths = {}, []
    for b, q0, m, s, tile, k0, k1, slot, run, runs, few, _ in rec:
        assert (q0, m, s) == (start[b], new[b], seq[b]) and few == (m * G <= 32) and (not few or tile == 0)
        seen.setdefault((b, tile), []).append((run, runs, k0, k1, slot))
        lengths.append((k1 - k0) * (3 if few else 8))
    for b in range(B):
        for tile in range(-(-new[b] * G // 256) if new[b] * G > 32 else 1):
            r = sorted(seen.pop((b, tile)))
            last = min((tile * 256 + 255) // G, new[b] - 1) if new[b] * G > 32 else new[b] - 1
            assert [x[0] for x in r] == list(range(r[0][1])) and len({x[4] for x in r}) == 1
            assert r[0][2] == 0 and r[-1][3] == -(-(seq[b] - new[b] + last + 1) // 64) and all(x[3] == y[2] for x, y in zip(r, r[1:]))
    assert not seen
    step = max(lengths) / 64 + 9                       # a bucket and the rounding of runs of one tile
    assert all(x >= y - step for x, y in zip(lengths, lengths[1:]))
    cut_tiles = {(b, t) for b, _, _, _, t, _, _, _, _, runs, few, _ in rec if runs > 1 and not few}
    assert cuts == len(cut_tiles) and {tuple(rec[i][[0, 4]]) for i in out[16:16 + cuts]} == cut_tiles
    slots = [(few, slot + run) for _, _, _, _, _, _, _, slot, run, runs, few, _ in rec if runs > 1]
    assert len(set(slots)) == len(slots) and all(x < 2 * z["side_by_side"] for _, x in slots)


def test_captured_and_replayed_with_other_lengths():
    """One graph of schedule and attention, replayed with other lengths, eager work and a synchronisation in between; a second
    graph shares its workspace."""
    b = Batch([500, 40, 333], [1, 60, 2], 8, 2, page=16, seed=15)
    c = ctx()
    b.buffers(c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b.schedule_call(c, s)
    b.attention_call(c, s)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            b.schedule_call(c, torch.cuda.current_stream())
            b.attention_call(c, torch.cuda.current_stream())
        graphs.append(g)
    full = list(b.seq)
    for cut in (0, 17, 250, 3):
        b.seq = [max(x - cut, n) for x, n in zip(full, b.new)]
        b.seq_d.copy_(ints(b.seq))
        for g in graphs:
            b.o.fill_(7)
            b.lse.fill_(7)
            g.replay()
            torch.cuda.synchronize()
            check_attention(b)
    tl.tl_ctx_destroy(c)


def test_two_streams_with_workspaces_of_their_own():
    bs = [Batch([2000, 9], [1, 1], 8, 2, seed=16), Batch([300], [200], 8, 2, seed=17)]
    c = ctx()
    streams = [torch.cuda.Stream() for _ in bs]
    for b in bs:
        b.buffers(c)
    torch.cuda.synchronize()
    for _ in range(3):
        for b, s in zip(bs, streams):
            b.schedule_call(c, s)
            b.attention_call(c, s)
    torch.cuda.synchronize()
    for b in bs:
        check_attention(b)
    tl.tl_ctx_destroy(c)
