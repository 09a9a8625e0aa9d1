"""A mixture-of-experts layer forward and backward by the calls a program makes in a row: against the gradients of the whole layer in 64
bits, and captured into a graph that is replayed with other tokens, another routing and other numbers of rows."""
import numpy as np
import pytest
import torch

import paper_2503_20313_amd as tl
from tests.moe_train_util import BF16, F32, I32, Lib, within

pytestmark = pytest.mark.gpu


class Layer:
    """out = x + sum_j w_j ((x W1_e) W2_e), e = the j-th expert of the token; loss gradient `dout` given."""

    def __init__(self, T, H, F, E, k, renormalize, room=1.0):
        self.T, self.H, self.F, self.E, self.k, self.renormalize = T, H, F, E, k, renormalize
        self.rows = max(1, int(T * k * room))
        d = dict(device="cuda")
        g = torch.Generator("cuda").manual_seed(T + H)
        self.x, self.dout = (torch.randn(T, H, generator=g, **d).to(BF16) for _ in range(2))
        self.logits = torch.randn(T, E, generator=g, **d)
        self.w1, self.w2 = (torch.randn(E, *s, generator=g, **d).mul(s[0] ** -0.5).to(BF16) for s in ((H, F), (F, H)))
        R, i = self.rows, lambda *s: torch.zeros(s, dtype=I32, **d)
        b, f = (lambda *s: torch.zeros(s, dtype=BF16, **d)), (lambda *s: torch.zeros(s, dtype=F32, **d))
        self.ids, self.w, self.tables = i(T, k), f(T, k), [i(E + 1), i(T * k), i(-(-T * k // 128) + E, 8), i(1)]
        self.off, self.sorted, self.pos = i(E + 1), i(T * k), i(T, k)
        self.xs, self.h, self.y, self.out = b(R, H), b(R, F), b(R, H), b(T, H)
        self.dy, self.dw, self.dh, self.dxs, self.dx = b(R, H), f(T, k), b(R, F), b(R, H), b(T, H)
        self.dw1, self.dw2, self.dlogits = b(E, H, F), f(E, F, H), f(T, E)

    def prepare(self, ctx):
        self.sort_bytes = tl.tl_moe_sort_query(ctx, self.T, self.k, self.E)
        n = max(tl.tl_moe_gemm_query(ctx, way, self.rows, a, b, self.E) for way in range(3) for a, b in ((self.H, self.F), (self.F, self.H)))
        self.sort_ws = torch.zeros(self.sort_bytes // 4, dtype=I32, device="cuda")
        self.ws = torch.full((n // 4,), -1, dtype=I32, device="cuda"), n
        torch.cuda.synchronize()

    def step(self, ctx, s):
        T, H, F, E, k, R = self.T, self.H, self.F, self.E, self.k, self.rows
        tl.tl_moe_route(ctx, self.logits, T, E, k, self.renormalize, 128, self.ids, self.w, *self.tables, s)
        tl.tl_moe_sort(ctx, self.ids, T, k, 0, E, self.off, self.sorted, self.pos, self.sort_ws, self.sort_bytes, s)
        tl.tl_moe_dispatch(ctx, self.x, self.pos, T, H, k, R, self.xs, s)
        tl.tl_moe_gemm(ctx, self.xs, self.w1, self.off, R, H, F, E, self.h, *self.ws, s)
        tl.tl_moe_gemm(ctx, self.h, self.w2, self.off, R, F, H, E, self.y, *self.ws, s)
        tl.tl_moe_combine(ctx, self.y, self.w, self.pos, T, H, k, R, self.x, self.out, s)
        tl.tl_moe_combine_grad(ctx, self.dout, self.y, self.w, self.pos, T, H, k, R, self.dy, self.dw, s)
        tl.tl_moe_route_grad(ctx, self.logits, self.ids, self.dw, T, E, k, self.renormalize, self.dlogits, s)
        tl.tl_moe_gemm_grad_w(ctx, self.h, self.dy, self.off, R, F, H, E, None, self.dw2, True, *self.ws, s)
        tl.tl_moe_gemm_grad_x(ctx, self.dy, self.w2, self.off, R, F, H, E, self.dh, *self.ws, s)
        tl.tl_moe_gemm_grad_w(ctx, self.xs, self.dh, self.off, R, H, F, E, None, self.dw1, False, *self.ws, s)
        tl.tl_moe_gemm_grad_x(ctx, self.dh, self.w1, self.off, R, H, F, E, self.dxs, *self.ws, s)
        tl.tl_moe_dispatch_grad(ctx, self.dxs, self.pos, T, H, k, R, self.dx, s)

    def results(self):
        return [t.clone() for t in (self.out, self.dx, self.dlogits, self.dw1, self.dw2, self.off, self.pos)]

    def exact(self):
        """Forward in 64 bits on the chosen experts, its gradients by differentiation (without those through the residual)."""
        x, l, w1, w2 = (t.double().cpu().requires_grad_(True) for t in (self.x, self.logits, self.w1, self.w2))
        ids = self.ids.long().cpu()
        if self.renormalize:
            w = torch.softmax(l.gather(1, ids), dim=1)
        else:
            w = torch.softmax(l, dim=1).gather(1, ids)
        here = (self.pos.cpu() >= 0) & (self.pos.cpu() < self.rows)
        out = torch.zeros(self.T, self.H, dtype=torch.float64)
        for e in range(self.E):
            t, j = torch.nonzero((ids == e) & here, as_tuple=True)
            out = out.index_add(0, t, w[t, j, None] * (x[t] @ w1[e] @ w2[e]))
        grads = torch.autograd.grad(out, (x, l, w1, w2), self.dout.double().cpu())
        return [out.detach() + x.detach(), *grads], self.bounds(w.detach(), ids, here)

    def bounds(self, w, ids, here):
        """How far rounding can take every result, step by step: a bf16 result is off by half a step u of its value (bounded by its
        terms' sizes), by what its inputs are off, carried on by the sizes of what they are multiplied with, and by a step of 32 bits a term, g.
        Products of two such errors are at most 2^-5 of them: the last factor."""
        u, g = 2.0 ** -8, 2.0 ** -23 * (max(self.H, self.F, self.T) + 64)
        x, dout, w1, w2 = (t.double().cpu().abs() for t in (self.x, self.dout, self.w1, self.w2))
        l = self.logits.double().cpu()
        ew = 2.0 ** -23 * (self.E + 32) * w                       # weights: a sum of E exponentials, arguments of a few units
        out, dx, dw, dw1, dw2 = u * x + g * x, torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(w1), torch.zeros_like(w2)
        val = lambda m: m.double().cpu().abs()
        for e in range(self.E):
            t, j = torch.nonzero((ids == e) & here, as_tuple=True)
            at = self.pos.cpu()[t, j].long()
            h, y, dy, dh, dxs = (val(m)[at] for m in (self.h, self.y, self.dy, self.dh, self.dxs))
            we, d = w[t, j, None], dout[t]
            eh = u * h + g * (x[t] @ w1[e])
            ey = u * y + eh @ w2[e] + g * (h @ w2[e])
            edy = u * dy + ew[t, j, None] * d
            edh = u * dh + edy @ w2[e].t() + g * (dy @ w2[e].t())
            edx = u * dxs + edh @ w1[e].t() + g * (dh @ w1[e].t())
            out.index_add_(0, t, we * ey + ew[t, j, None] * y + (u + g) * we * y)
            dx.index_add_(0, t, edx + (u + g) * dxs)
            dw[t, j] = (d * ey).sum(1) + g * (d * y).sum(1)
            dw1[e] = x[t].t() @ edh + (u + g) * (x[t].t() @ dh)
            dw2[e] = h.t() @ edy + eh.t() @ dy + (u + g) * (h.t() @ dy)
        share = torch.zeros_like(l).scatter_(1, ids, w) if self.renormalize else torch.softmax(l, 1)
        chosen = torch.zeros_like(l).scatter_(1, ids, 1.0)
        e_dw = dw + g * self.dw.double().cpu().abs() * 4
        dl = torch.zeros_like(l).scatter_(1, ids, w * e_dw) + share * (w * e_dw).sum(1, keepdim=True) + 2.0 ** -24 * chosen
        return [1.05 * b for b in (out, dx, dl, dw1, dw2)]


# a layer as it is trained, one token, a full buffer, few rows of many experts
SHAPES = [(300, 256, 136, 8, 2, True, 1.0), (1, 64, 72, 4, 2, False, 1.0), (200, 128, 64, 16, 3, True, 0.8), (48, 512, 264, 32, 5, False, 1.0)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_step_against_the_layer_in_64_bits(shape):
    layer = Layer(*shape)
    with Lib() as ctx:
        layer.prepare(ctx)
        layer.step(ctx, torch.cuda.current_stream())
        torch.cuda.synchronize()
        refs, bounds = layer.exact()
        for name, got, ref, bound in zip(("out", "dx", "dlogits", "dw1", "dw2"), layer.results(), refs, bounds):
            within(got.double().cpu().numpy(), ref.numpy(), bound.numpy(), name)


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_step_captured_and_replayed(shape):
    layer = Layer(*shape)
    with Lib() as ctx:
        layer.prepare(ctx)
        s = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            layer.step(ctx, s)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            layer.step(ctx, s)
        for replay in range(4):
            g = torch.Generator("cuda").manual_seed(replay)
            layer.x.copy_(torch.randn(layer.x.shape, device="cuda", generator=g))
            layer.logits.copy_(torch.randn(layer.logits.shape, device="cuda", generator=g) + 3.0 * replay * (torch.arange(layer.E, device="cuda") == replay))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            got = layer.results()
            layer.step(ctx, torch.cuda.current_stream())
            torch.cuda.synchronize()
            for a, b in zip(got, layer.results()):
                assert torch.equal(a, b)


def test_two_layers_side_by_side():
    """Two programs' worth of buffers and workspaces on two streams at once."""
    layers = [Layer(*SHAPES[0]), Layer(*SHAPES[3])]
    with Lib() as ctx:
        for layer in layers:
            layer.prepare(ctx)
            layer.step(ctx, torch.cuda.current_stream())
        torch.cuda.synchronize()
        alone = [layer.results() for layer in layers]
        streams = [torch.cuda.Stream() for _ in layers]
        torch.cuda.synchronize()
        for _ in range(5):
            for layer, s in zip(layers, streams):
                layer.step(ctx, s)
        torch.cuda.synchronize()
        for layer, ref in zip(layers, alone):
            for a, b in zip(layer.results(), ref):
                assert torch.equal(a, b)
