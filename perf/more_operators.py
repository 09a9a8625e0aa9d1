"""The operators of a mixture-of-experts layer in training, as data: which calls, at which sizes, on which inputs, and their plain forms.

tl_moe_route chooses the experts of every token; row (t, j), number t*topk + j, is token t at its j-th expert.  Then

  sort         tl_moe_sort: the rows in the order of their experts, and for every row its place in it
  dispatch     tl_moe_dispatch, tl_moe_dispatch_grad: token rows into that order, and the gradient back
  products     tl_moe_gemm, tl_moe_gemm_grad_x, tl_moe_gemm_grad_w: every expert's product on its rows, and both gradients
  combine      tl_moe_combine, tl_moe_combine_grad: rows back to their tokens with their weights, and the gradients of rows and weights
  route_grad   tl_moe_route_grad: the gradient of the gate's logits from that of the weights

With `own` false a pass is the plain form: elementary torch operations in 32 bits, rounded once.  With `own` true it is the
calls a program makes of the library.  Matrices are bf16, logits, weights and their gradients fp32.
"""
import math
import random

import torch

own = False

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32


# ---------------------------------------------------------------------------------------------------------------------
# The cases.  T tokens of H features, topk experts each out of `E * ranks`, of which this rank holds E; in `products`, `rows` rows
# spread over E experts by shares that `spread` picks (0: even).  `room`: rows of the sorted matrices, as a share of T*topk.
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # One token being decoded: the smallest call, latency alone.
        dict(name="sort token", op="sort", T=1, topk=2, E=8, ranks=1),
        # A whole training batch with many experts: the longest lists.
        dict(name="sort batch", op="sort", T=16381, topk=8, E=64, ranks=1),
        # The router of a small batch, weights normalised over the chosen experts.
        dict(name="route_grad small", op="route_grad", T=512, topk=5, E=32, renormalize=True),
        # The router of a training batch, softmax weights as they are.
        dict(name="route_grad batch", op="route_grad", T=16384, topk=8, E=64, renormalize=False),
        # A training batch of the benchmark's top-5 layer into its experts' order.
        dict(name="dispatch batch", op="dispatch", dir="forward", T=8192, H=4096, topk=5, E=32, ranks=1, room=1),
        # The gradient back on a rank that holds a quarter of the experts; odd sizes, most tokens have one row here, or none.
        dict(name="dispatch grad share", op="dispatch", dir="grad", T=8191, H=2056, topk=5, E=8, ranks=4, room=1),
        # One token being decoded, the residual added: latency alone.
        dict(name="combine token", op="combine", dir="forward", T=1, H=4096, topk=2, E=32, ranks=1, room=1, add=True),
        # The gradients of a training batch: every matrix of the layer's output side is read or written once.
        dict(name="combine grad batch", op="combine", dir="grad", T=8192, H=4096, topk=5, E=32, ranks=1, room=1, add=False),
        # A decode step of 64 requests, top-5 of 32 small experts: bound by the reading of the experts' weights.
        dict(name="products decode", op="products", dir="forward", rows=320, K=2048, N=1536, E=32, spread=1),
        # The gradient of the rows of a training batch with few, unevenly used experts.
        dict(name="products grad_x batch", op="products", dir="grad_x", rows=16384, K=4096, N=2048, E=8, spread=2),
        # The gradient of the weights with many experts: some hundred rows each, as much to store as to multiply.
        dict(name="products grad_w batch", op="products", dir="grad_w", rows=16384, K=4096, N=1792, E=32, spread=3, accumulate=False),
        # The same into accumulators in fp32, smaller layer, rows that are not a multiple of anything.
        dict(name="products grad_w accumulate", op="products", dir="grad_w", rows=16001, K=2048, N=1536, E=8, spread=4, accumulate=True),
    ]


def _log_int(rng, lo, hi):
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


def draw(rng):
    op = rng.choice(["sort", "route_grad", "dispatch", "dispatch", "combine", "combine", "products", "products", "products"])
    E = rng.choice([2, 4, 8, 8, 16, 32, 32, 60, 64, 128, 256])
    topk = min(rng.choice([1, 2, 2, 4, 5, 6, 8]), E)
    ranks = rng.choice([1, 1, 1, 2, 4])
    if op == "sort":
        return dict(op=op, T=_log_int(rng, 1, 16384), topk=topk, E=E, ranks=ranks)
    if op == "route_grad":
        return dict(op=op, T=_log_int(rng, 1, min(16384, 16384 * 64 // E)), topk=topk, E=E, renormalize=rng.random() < 0.5)
    if op in ("dispatch", "combine"):
        H = 8 * _log_int(rng, 16, 1024)
        T = _log_int(rng, 1, min(16384, 8192 * 5 * 4096 // (H * topk)))
        c = dict(op=op, dir=rng.choice(["forward", "grad"]), T=T, H=H, topk=topk, E=E, ranks=ranks, room=rng.choice([1, 1, 1, 0.75]))
        return c if op == "dispatch" else dict(c, add=c["dir"] == "forward" and rng.random() < 0.5)
    K, N = 8 * _log_int(rng, 16, 1024), 8 * _log_int(rng, 16, 1024)
    while E * K * N > 32 * 4096 * 1792:
        E //= 2
    rows = _log_int(rng, 1, min(65536, 16384 * 4096 * 1792 // (K * N)))
    way = rng.choice(["forward", "grad_x", "grad_w"])
    c = dict(op=op, dir=way, rows=rows, K=K, N=N, E=E, spread=rng.choice([0, rng.randrange(1, 1 << 20)]))
    if way == "grad_w":
        c["accumulate"] = rng.random() < 0.5 and E * K * N <= 8 * 4096 * 1792
    return c


def _counts(case):
    """Rows of every expert."""
    rng = random.Random(case["spread"])
    E, rows = case["E"], case["rows"]
    shares = [math.exp(rng.gauss(0, 0.7)) if case["spread"] else 1.0 for _ in range(E)]
    if case["spread"] and E > 2:
        shares[rng.randrange(E)] = 0.0                  # one that nobody chose
    at = [0.0]
    for s in shares:
        at.append(at[-1] + s)
    cut = [int(round(a / at[-1] * rows)) for a in at]
    return [b - a for a, b in zip(cut, cut[1:])]


# ---------------------------------------------------------------------------------------------------------------------
# What a program has in hand before the call
# ---------------------------------------------------------------------------------------------------------------------
class _Draw:
    def __init__(self, seed):
        self.dev = torch.device("cuda", torch.cuda.current_device())
        self.g = torch.Generator(device=self.dev)
        self.g.manual_seed(seed)

    def normal(self, *shape, dtype=BF16, scale=1.0):
        x = torch.empty(shape, device=self.dev, dtype=dtype)
        return x.normal_(0.0, scale, generator=self.g)

    def zeros(self, *shape, dtype=BF16):
        return torch.zeros(shape, device=self.dev, dtype=dtype)


class _Context:
    """The library's context of this program."""

    def __init__(self):
        import paper_2503_20313_amd as tl
        self.tl = tl
        self.ctx = tl.tl_ctx_create(world_size=1, rank=0, channels_per_rank=1, comm_mode=tl.TL_COMM_NONE)

    def __del__(self):
        if getattr(self, "ctx", None) is not None:
            self.tl.tl_ctx_destroy(self.ctx)
            self.ctx = None


def _gate(d, T, E, topk):
    """Logits of a gate that likes some experts better than others, the chosen experts and their softmax."""
    logits = d.normal(T, E, dtype=F32) + d.normal(E, dtype=F32, scale=0.5)
    p, ids = torch.softmax(logits, dim=1).topk(topk, dim=1)
    return logits, ids.to(I32), p


def _sorted_maps(ids, first, E):
    """(expert of every row in their order, row numbers in that order, rows that take part) of the rows whose expert is one of ours."""
    e = ids.flatten().long() - first
    e = torch.where((e >= 0) & (e < E), e, E)
    key, order = torch.sort(e, stable=True)
    return key, order, e < E


def prepare(case, seed):
    d, op = _Draw(seed), case["op"]
    s = {"case": case}
    if own:
        s["lib"] = _Context()
    if op == "products":
        rows, K, N, E = case["rows"], case["K"], case["N"], case["E"]
        s["counts"] = _counts(case)
        s["offsets"] = torch.tensor([0] + s["counts"], device=d.dev).cumsum(0).to(I32)
        if case["dir"] != "grad_x":
            s["x"] = d.normal(rows, K)
        if case["dir"] != "forward":
            s["dy"] = d.normal(rows, N, scale=0.1)
        if case["dir"] == "grad_w":
            s["add"] = d.normal(E, K, N, dtype=F32) if case["accumulate"] else None
            s["out"] = d.zeros(E, K, N, dtype=F32 if case["accumulate"] else BF16)
        else:
            s["w"] = d.normal(E, K, N, scale=0.02)
            s["out"] = d.zeros(rows, N if case["dir"] == "forward" else K)
        if own:
            tl = s["lib"].tl
            way = dict(forward=tl.TL_MOE_FORWARD, grad_x=tl.TL_MOE_GRAD_X, grad_w=tl.TL_MOE_GRAD_W)[case["dir"]]
            s["ws_bytes"] = tl.tl_moe_gemm_query(s["lib"].ctx, way, rows, K, N, E)
            s["ws"] = d.zeros(s["ws_bytes"] // 4, dtype=I32)
        return s
    T, topk, E = case["T"], case["topk"], case["E"]
    ranks = case.get("ranks", 1)
    logits, ids, p = _gate(d, T, E * ranks, topk)
    if op == "route_grad":
        s["logits"], s["ids"] = logits, ids
        s["dw"], s["dlogits"] = d.normal(T, topk, dtype=F32), d.zeros(T, E, dtype=F32)
        return s
    first = E * (ranks // 2)                             # a rank in the middle
    if op == "sort":
        s["ids"], s["first"] = ids, first
        s["offsets"], s["sorted_row"], s["row_pos"] = d.zeros(E + 1, dtype=I32), d.zeros(T * topk, dtype=I32), d.zeros(T, topk, dtype=I32)
        if own:
            s["ws_bytes"] = s["lib"].tl.tl_moe_sort_query(s["lib"].ctx, T, topk, E)
            s["ws"] = d.zeros(s["ws_bytes"] // 4, dtype=I32)
        return s
    H = case["H"]
    rows = s["rows"] = max(1, int(T * topk * case["room"]))
    _, order, part = _sorted_maps(ids, first, E)
    pos = torch.empty_like(order)
    pos[order] = torch.arange(T * topk, device=d.dev)
    s["row_pos"] = torch.where(part, pos, -1).to(I32).reshape(T, topk)
    if op == "combine":
        s["w"] = (p / p.sum(1, keepdim=True)).contiguous()
    if op == "dispatch" and case["dir"] == "forward":
        s["x"], s["out"] = d.normal(T, H), d.zeros(rows, H)
    elif op == "dispatch":
        s["dxs"], s["out"] = d.normal(rows, H, scale=0.1), d.zeros(T, H)
    else:
        s["ys"] = d.normal(rows, H)
        if case["dir"] == "forward":
            s["add"] = d.normal(T, H) if case["add"] else None
            s["out"] = d.zeros(T, H)
        else:
            s["dout"] = d.normal(T, H, scale=0.1)
            s["dys"], s["dw"] = d.zeros(rows, H), d.zeros(T, topk, dtype=F32)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# One pass: the library's calls
# ---------------------------------------------------------------------------------------------------------------------
def _own(s):
    c, tl, ctx = s["case"], s["lib"].tl, s["lib"].ctx
    stream = torch.cuda.current_stream()
    op, way = c["op"], c.get("dir")
    if op == "sort":
        tl.tl_moe_sort(ctx, s["ids"], c["T"], c["topk"], s["first"], c["E"], s["offsets"], s["sorted_row"], s["row_pos"], s["ws"], s["ws_bytes"], stream)
    elif op == "route_grad":
        tl.tl_moe_route_grad(ctx, s["logits"], s["ids"], s["dw"], c["T"], c["E"], c["topk"], c["renormalize"], s["dlogits"], stream)
    elif op == "products":
        sizes, ws = (s["offsets"], c["rows"], c["K"], c["N"], c["E"]), (s["ws"], s["ws_bytes"], stream)
        if way == "forward":
            tl.tl_moe_gemm(ctx, s["x"], s["w"], *sizes, s["out"], *ws)
        elif way == "grad_x":
            tl.tl_moe_gemm_grad_x(ctx, s["dy"], s["w"], *sizes, s["out"], *ws)
        else:
            tl.tl_moe_gemm_grad_w(ctx, s["x"], s["dy"], *sizes, s["add"], s["out"], c["accumulate"], *ws)
    else:
        sizes = (s["row_pos"], c["T"], c["H"], c["topk"], s["rows"])
        if op == "dispatch" and way == "forward":
            tl.tl_moe_dispatch(ctx, s["x"], *sizes, s["out"], stream)
        elif op == "dispatch":
            tl.tl_moe_dispatch_grad(ctx, s["dxs"], *sizes, s["out"], stream)
        elif way == "forward":
            tl.tl_moe_combine(ctx, s["ys"], s["w"], *sizes, s["add"], s["out"], stream)
        else:
            tl.tl_moe_combine_grad(ctx, s["dout"], s["ys"], s["w"], *sizes, s["dys"], s["dw"], stream)


# ---------------------------------------------------------------------------------------------------------------------
# One pass: the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _plain_sort(s):
    E, n = s["case"]["E"], s["ids"].numel()
    key, order, part = _sorted_maps(s["ids"], s["first"], E)
    at = torch.arange(n, device=key.device)
    s["offsets"].copy_(torch.searchsorted(key, torch.arange(E + 1, device=key.device)))
    s["sorted_row"].copy_(torch.where(key < E, order, s["sorted_row"].long()))
    pos = torch.empty_like(order)
    pos[order] = at
    s["row_pos"].copy_(torch.where(part, pos, -1).reshape(s["row_pos"].shape))


def _plain_route_grad(s):
    l, ids, g = s["logits"], s["ids"].long(), s["dw"]
    p = torch.exp(l - l.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    w = p.gather(1, ids)
    if s["case"]["renormalize"]:
        w = w / w.sum(1, keepdim=True)
        dl = torch.zeros_like(l).scatter_add(1, ids, w * (g - (w * g).sum(1, keepdim=True)))
    else:
        dl = p * (torch.zeros_like(l).scatter_add(1, ids, g) - (w * g).sum(1, keepdim=True))
    s["dlogits"].copy_(dl)


def _rows_of(s, m):
    """Row (t, j) of a sorted matrix in 32 bits, for one j after the other; zeros where it takes no part."""
    for j in range(s["case"]["topk"]):
        pos = s["row_pos"][:, j].long()
        here = (pos >= 0) & (pos < s["rows"])
        yield j, here, torch.where(here[:, None], m[torch.where(here, pos, 0)].to(F32), 0.0)


def _plain_rows(s):
    c = s["case"]
    if c["dir"] == "forward":
        if c["op"] == "dispatch":
            for j in range(c["topk"]):
                pos = s["row_pos"][:, j].long()
                here = (pos >= 0) & (pos < s["rows"])
                s["out"][pos[here]] = s["x"][here]
            return
        y = s["out"].new_zeros(s["out"].shape, dtype=F32) if s["add"] is None else s["add"].to(F32)
        for j, here, row in _rows_of(s, s["ys"]):
            y = y + torch.where(here, s["w"][:, j], 0.0)[:, None] * row
        s["out"].copy_(y)
    elif c["op"] == "dispatch":
        y = s["out"].new_zeros(s["out"].shape, dtype=F32)
        for _, _, row in _rows_of(s, s["dxs"]):
            y = y + row
        s["out"].copy_(y)
    else:
        dout = s["dout"].to(F32)
        for j, here, row in _rows_of(s, s["ys"]):
            s["dys"][s["row_pos"][:, j].long()[here]] = (s["w"][:, j, None] * dout)[here].to(BF16)
            s["dw"][:, j] = (dout * row).sum(1)


def _plain_products(s):
    c, lo = s["case"], 0
    for e, n in enumerate(s["counts"]):
        rows = slice(lo, lo + n)
        lo += n
        if c["dir"] == "forward":
            s["out"][rows] = (s["x"][rows].to(F32) @ s["w"][e].to(F32)).to(BF16)
        elif c["dir"] == "grad_x":
            s["out"][rows] = (s["dy"][rows].to(F32) @ s["w"][e].to(F32).t()).to(BF16)
        else:
            dw = s["x"][rows].to(F32).t() @ s["dy"][rows].to(F32)
            s["out"][e] = dw if s["add"] is None else s["add"][e] + dw


_OUTPUTS = dict(sort=("offsets", "sorted_row", "row_pos"), route_grad=("dlogits",), products=("out",), dispatch=("out",), combine=("out",))


def _outputs(c):
    return ("dys", "dw") if c["op"] == "combine" and c["dir"] == "grad" else _OUTPUTS[c["op"]]


def run(s):
    c = s["case"]
    if own:
        _own(s)
    else:
        dict(sort=_plain_sort, route_grad=_plain_route_grad, products=_plain_products, dispatch=_plain_rows, combine=_plain_rows)[c["op"]](s)
    return {x: s[x] for x in _outputs(c)}


# ---------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_route_grad(s):
    """The gradient of <dw, weights(logits)>, by differentiating the weights' definition."""
    c, l = s["case"], s["logits"].double().requires_grad_(True)
    with torch.enable_grad():
        chosen = l.gather(1, s["ids"].long())
        w = torch.exp(chosen - torch.logsumexp(chosen if c["renormalize"] else l, dim=1, keepdim=True))
        return torch.autograd.grad(w, l, s["dw"].double())[0]


def _exact_rows(s):
    """Over the list of (token, choice, place) that take part."""
    c = s["case"]
    pos = s["row_pos"].long()
    t, j = torch.nonzero((pos >= 0) & (pos < s["rows"]), as_tuple=True)
    at = pos[t, j]
    grad = c["dir"] == "grad"
    if c["op"] == "dispatch" and not grad:
        return {"out": torch.zeros(s["out"].shape, dtype=F64, device=t.device).index_copy_(0, at, s["x"].double()[t])}
    if not grad or c["op"] == "dispatch":
        out = torch.zeros(s["out"].shape, dtype=F64, device=t.device) if s.get("add") is None else s["add"].double()
        for k in range(c["topk"]):                       # (a token has one row per choice: no two go to one place)
            m = j == k
            rows = s["dxs"].double()[at[m]] if c["op"] == "dispatch" else s["ys"].double()[at[m]] * s["w"].double()[t[m], k, None]
            out[t[m]] += rows
        return {"out": out}
    dys, dw = torch.zeros(s["dys"].shape, dtype=F64, device=t.device), torch.zeros(s["dw"].shape, dtype=F64, device=t.device)
    for k in range(c["topk"]):
        m = j == k
        dout = s["dout"].double()[t[m]]
        dys[at[m]] = dout * s["w"].double()[t[m], k, None]
        dw[t[m], k] = (dout * s["ys"].double()[at[m]]).sum(1)
    return {"dys": dys, "dw": dw}


def _exact_products(s):
    c = s["case"]
    out = torch.zeros(s["out"].shape, dtype=F64, device=s["out"].device)
    if c["dir"] == "grad_w" and s["add"] is not None:
        out += s["add"]
    end = s["offsets"].tolist()
    for e in range(c["E"]):
        lo, hi = end[e], end[e + 1]
        if lo == hi:
            continue
        if c["dir"] == "grad_w":
            out[e].addmm_(s["x"][lo:hi].double().t().contiguous(), s["dy"][lo:hi].double())
        elif c["dir"] == "forward":
            torch.matmul(s["x"][lo:hi].double(), s["w"][e].double(), out=out[lo:hi])
        else:
            torch.matmul(s["dy"][lo:hi].double(), s["w"][e].double().t().contiguous(), out=out[lo:hi])
    return {"out": out}


def exact(case, seed):
    if case["op"] == "sort":
        return None                     # whole numbers
    s = prepare(case, seed)
    with torch.no_grad():
        if case["op"] == "route_grad":
            return {"dlogits": _exact_route_grad(s)}
        return _exact_products(s) if case["op"] == "products" else _exact_rows(s)


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "products":
        rows, K, N, E = case["rows"], case["K"], case["N"], case["E"]
        if case["dir"] == "grad_w":
            weights = E * K * N * (8.0 if case["accumulate"] else 2.0)
        else:
            weights = 2.0 * K * N * sum(n > 0 for n in _counts(case))
        return {"bytes": 2.0 * rows * (K + N) + weights + 4.0 * (E + 1), "flops": 2.0 * rows * K * N}
    n = case["T"] * case["topk"]
    if op == "route_grad":
        return {"bytes": 8.0 * case["T"] * case["E"] + 8.0 * n, "flops": 6.0 * case["T"] * case["E"] + 4.0 * n}
    here = n / case["ranks"]            # rows whose expert is one of this rank's: that many in the mean
    if op == "sort":
        return {"bytes": 4.0 * (2 * n + here + case["E"] + 1), "flops": 0.0}
    T, H = case["T"], case["H"]
    here = min(here, n * case["room"])
    if op == "dispatch":
        return {"bytes": 2.0 * (T + here) * H + 4.0 * n, "flops": 0.0 if case["dir"] == "forward" else here * H}
    if case["dir"] == "forward":
        return {"bytes": 2.0 * (T * (2 if case["add"] else 1) + here) * H + 8.0 * n, "flops": 2.0 * here * H}
    return {"bytes": 2.0 * (T + 2 * here) * H + 12.0 * n, "flops": 3.0 * here * H}
