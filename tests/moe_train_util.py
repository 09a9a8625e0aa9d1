"""Helpers of the tests of a mixture-of-experts layer in training: tensors, routings, bounds."""
import numpy as np
import torch

import paper_2503_20313_amd as tl
from oracle import moe_train as o

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
HALF16 = 2.0 ** -8        # half a step of bf16, relative
HALF32 = 2.0 ** -24


class Lib:
    """A context of its own, as a program has one."""

    def __init__(self):
        self.ctx = tl.tl_ctx_create(world_size=1, rank=0, channels_per_rank=1, comm_mode=tl.TL_COMM_NONE)

    def __enter__(self):
        return self.ctx

    def __exit__(self, *_):
        torch.cuda.synchronize()
        tl.tl_ctx_destroy(self.ctx)


def gpu(a, dtype):
    return torch.as_tensor(np.asarray(a)).to(dtype).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def bf16_normal(rng, *shape, scale=1.0):
    """bf16 values, as a device tensor and in 64 bits."""
    t = torch.from_numpy(rng.normal(size=shape).astype(np.float32) * np.float32(scale)).to(BF16)
    return t.cuda(), t.double().numpy()


def small_ints(rng, *shape):
    """Values whose products and sums are exact in fp32."""
    a = rng.integers(-2, 3, size=shape)
    return gpu(a, BF16), a.astype(np.float64)


def choose(rng, T, E, k):
    """k different experts for every token, some liked better than others."""
    score = rng.normal(size=(T, E)) + rng.normal(size=E)
    return np.argsort(-score, axis=1, kind="stable")[:, :k].astype(np.int64)


def places(rng, T, k, E=8, ranks=1):
    """row_pos of a routing: this rank's experts are the middle ones of E * ranks."""
    return o.sort_rows(choose(rng, T, E * ranks, k), E * (ranks // 2), E)


def rounded(ref, slack):
    """Bound on a bf16 result of a value that fp32 arithmetic has to `slack`."""
    return HALF16 * (np.abs(ref) + slack) + slack


def within(got, ref, bound, what=""):
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} outside, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {ref[bad][0]} +- {np.broadcast_to(bound, ref.shape)[bad][0]}"


def sort_call(ctx, ids, first, E, stream=None, ws=None):
    """ids on the device -> offsets, sorted_row, row_pos (poisoned with -7 beforehand)."""
    T, k = ids.shape
    off, rows, pos = (torch.full(s, -7, dtype=I32, device="cuda") for s in ((E + 1,), (T * k,), (T, k)))
    n = tl.tl_moe_sort_query(ctx, T, k, E)
    if ws is None:
        ws = torch.full((n // 4,), -1, dtype=I32, device="cuda")
    tl.tl_moe_sort(ctx, ids, T, k, first, E, off, rows, pos, ws, n, stream)
    return off, rows, pos


def product_ws(ctx, way, rows, K, N, E):
    n = tl.tl_moe_gemm_query(ctx, way, rows, K, N, E)
    return torch.full((n // 4,), -1, dtype=I32, device="cuda"), n        # needs no preparation
