"""The operators of a serving step over a paged cache, as data: which calls, at which sizes, on which inputs, and their plain forms.

Between the projection that makes queries, keys and values (tl_ag_gemm) and the one that follows the attention (tl_gemm_rs), a step runs

  slots            tl_paged_slots: block tables, slots, positions and row offsets of a batch, from the requests' lengths
  norm_rope        tl_qk_norm_rope: RMS norm of every query and key head and the position rotation, in one pass
  norm_rope_cache  tl_qk_norm_rope_cache: the same, with keys and values stored in the pages of the cache
  attention        tl_paged_schedule + tl_paged_attention: attention of the new tokens over the cached keys
  step             all of these in a row

With `own` false a pass is the plain form: elementary torch operations in 32 bits, rounded once.  With `own` true it is the
calls a program makes of the library.  bf16 tensors, head_dim 128, heads = one rank's share of a tensor-parallel layer.
"""
import math
import random

import torch

own = False

D = 128                 # head_dim
EPS = 1e-6
SCALE = D ** -0.5
BF16, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64


# ---------------------------------------------------------------------------------------------------------------------
# The cases.  B requests; `chunks` of them bring n_lo..n_hi new tokens, the others one each; c_lo..c_hi tokens of a request
# are in the cache already; `lens` picks the lengths.
# ---------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # One decode step of a serving batch: one new token per request, latency alone.
        dict(name="slots decode", op="slots", B=64, chunks=0, n_lo=1, n_hi=1, c_lo=100, c_hi=4000, page=16, lens=1),
        # A large batch of prompts admitted at once, ragged, small pages: the longest tables and maps.
        dict(name="slots prefill", op="slots", B=512, chunks=512, n_lo=1, n_hi=250, c_lo=0, c_hi=2000, page=16, lens=2),
        # A single token of one request, rotation in neighbouring pairs: the smallest call.
        dict(name="norm_rope token", op="norm_rope", T=1, heads_q=32, heads_kv=8, rot=128, pairs="neighbours", norm=True),
        # The query and key shard of the long-context attention benchmark (32768 positions over 8 ranks, 32 heads).
        dict(name="norm_rope shard", op="norm_rope", T=4096, heads_q=32, heads_kv=32, rot=128, pairs="halves", norm=True),
        # A decode step of 64 requests, one rank of eight of a 64/8-head layer, rows of a packed projection.
        dict(name="norm_rope_cache decode", op="norm_rope_cache", T=64, heads_q=8, heads_kv=1, rot=128, pairs="halves", norm=True, page=16),
        # A prompt batch of ragged length with a partial rotation, all heads of a 32/8-head layer.
        dict(name="norm_rope_cache prefill", op="norm_rope_cache", T=8001, heads_q=32, heads_kv=8, rot=64, pairs="halves", norm=True, page=64),
        # One request, one token, a short context: the smallest attention call.
        dict(name="attention token", op="attention", B=1, chunks=0, n_lo=1, n_hi=1, c_lo=1000, c_hi=1000, heads_q=8, heads_kv=1, page=16, window=0, lens=3),
        # A decode batch with ragged contexts, small pages: bound by the reading of the cache.
        dict(name="attention decode batch", op="attention", B=64, chunks=0, n_lo=1, n_hi=1, c_lo=500, c_hi=8000, heads_q=32, heads_kv=8, page=16, window=0, lens=4),
        # One very long request: few rows, a long axis to split.
        dict(name="attention decode long", op="attention", B=1, chunks=0, n_lo=1, n_hi=1, c_lo=130000, c_hi=130000, heads_q=32, heads_kv=8, page=64, window=0, lens=5),
        # A whole prompt without anything cached: bound by the matrix products.
        dict(name="attention prompt", op="attention", B=1, chunks=1, n_lo=8192, n_hi=8192, c_lo=0, c_hi=0, heads_q=32, heads_kv=8, page=64, window=0, lens=6),
        # The next chunk of a long prompt, odd sizes: few query tiles, a long axis.
        dict(name="attention chunk", op="attention", B=1, chunks=1, n_lo=509, n_hi=509, c_lo=31003, c_hi=31003, heads_q=16, heads_kv=2, page=32, window=0, lens=7),
        # A whole mixed step: 40 decoding requests and 8 prompt chunks, a sliding window, five query heads to a key head.
        dict(name="step mixed", op="step", B=48, chunks=8, n_lo=100, n_hi=256, c_lo=200, c_hi=4000, heads_q=20, heads_kv=4, rot=128, pairs="halves", norm=True,
             page=16, window=2048, lens=8),
    ]


def _log_int(rng, lo, hi):
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


def draw(rng):
    op = rng.choice(["slots", "norm_rope", "norm_rope_cache", "attention", "attention", "attention", "step"])
    page = rng.choice([16, 16, 32, 64, 128])
    kv = rng.choice([1, 1, 2, 4, 8])
    heads = dict(heads_q=kv * rng.choice([1, 2, 4, 5, 8, 16] if kv <= 2 else [1, 2, 4, 5]), heads_kv=kv)
    rotation = dict(rot=rng.choice([128, 128, 64, 32]), pairs=rng.choice(["halves", "halves", "neighbours"]), norm=rng.random() < 0.8)
    lens = rng.randrange(1 << 20)
    if op == "slots":
        B = _log_int(rng, 1, 512)
        n = _log_int(rng, 1, 250)
        chunks = rng.choice([0, B, rng.randrange(B + 1)])
        return dict(op=op, B=B, chunks=chunks, n_lo=1, n_hi=n, c_lo=0, c_hi=_log_int(rng, 10, 8000), page=page, lens=lens)
    if op in ("norm_rope", "norm_rope_cache"):
        T = _log_int(rng, 1, 8001)
        c = dict(op=op, T=T, **heads, **rotation)
        return c if op == "norm_rope" else dict(c, page=page)
    window = rng.choice([0, 0, 0, 128, 1000])
    kind = rng.choice(["decode", "decode", "chunk", "mixed"])
    if kind == "decode":
        B = _log_int(rng, 1, 128)
        c_hi = _log_int(rng, 16, min(130000, 360000 * 8 // (B * kv)))
        c = dict(op=op, B=B, chunks=0, n_lo=1, n_hi=1, c_lo=c_hi // rng.choice([1, 2, 10]), c_hi=c_hi)
    elif kind == "chunk":
        n = _log_int(rng, 2, 4096)
        c_hi = _log_int(rng, 1, max(1, min(32000, 16000000 // n)))
        c = dict(op=op, B=1, chunks=1, n_lo=n, n_hi=n, c_lo=c_hi, c_hi=c_hi)
    else:
        B = _log_int(rng, 2, 64)
        c = dict(op=op, B=B, chunks=rng.randrange(1, max(2, B // 4)), n_lo=2, n_hi=_log_int(rng, 2, 400), c_lo=0, c_hi=_log_int(rng, 16, 4000))
    c = dict(c, **heads, page=page, window=window, lens=lens)
    return dict(c, **rotation) if op == "step" else c


def _lengths(case):
    """(cached tokens, new tokens) of every request."""
    rng = random.Random(case["lens"])
    new = [rng.randint(case["n_lo"], case["n_hi"]) if i < case["chunks"] else 1 for i in range(case["B"])]
    rng.shuffle(new)
    return [rng.randint(case["c_lo"], case["c_hi"]) for _ in new], new


# ---------------------------------------------------------------------------------------------------------------------
# What a program has in hand before the call
# ---------------------------------------------------------------------------------------------------------------------
class _Draw:
    def __init__(self, seed):
        self.dev = torch.device("cuda", torch.cuda.current_device())
        self.g = torch.Generator(device=self.dev)
        self.g.manual_seed(seed)

    def normal(self, *shape, dtype=BF16):
        return torch.randn(shape, generator=self.g, device=self.dev, dtype=dtype)

    def perm(self, n):
        return torch.randperm(n, generator=self.g, device=self.dev).to(I32)

    def ints(self, values):
        return torch.tensor(values, dtype=I32, device=self.dev)

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


def _pages(n, page):
    return -(-n // page)


def _prepare_requests(d, case, s):
    """Lengths, a pool of pages in random order, the block table of what is cached already, and the free list."""
    ctx, new = _lengths(case)
    P = case["page"]
    s["ctx"], s["new"] = ctx, new
    s["ctx_lens"], s["new_lens"] = d.ints(ctx), d.ints(new)
    have = [_pages(c, P) for c in ctx]
    need = [_pages(c + n, P) for c, n in zip(ctx, new)]
    s["max_blocks"] = max(need)
    s["n_pages"] = sum(need) + 8
    order = d.perm(s["n_pages"])
    table = d.zeros(case["B"], s["max_blocks"], dtype=I32)
    if case["op"] == "attention":       # the new tokens are in the cache already: every page is in the table
        have = need
    cut = torch.tensor([0] + have).cumsum(0).tolist()
    for b in range(case["B"]):
        table[b, :have[b]] = order[cut[b]:cut[b + 1]]
    s["table"] = table
    s["free"] = order[cut[-1]:].contiguous()
    s["T"] = sum(new)


def _prepare_slots(d, case, s):
    B, T = case["B"], s["T"]
    s["free_from"], s["free_to"] = d.zeros(1, dtype=I32), d.zeros(1, dtype=I32)
    s["query_start"], s["seq_lens"] = d.zeros(B + 1, dtype=I32), d.zeros(B, dtype=I32)
    s["slots"], s["positions"], s["counts"] = d.zeros(T, dtype=I32), d.zeros(T, dtype=I32), d.zeros(4, dtype=I32)


def _prepare_rows(d, case, s, T, max_position):
    """The rows of a packed projection, norm weights and the table of angles."""
    Hq, Hk = case["heads_q"], case["heads_kv"]
    s["qkv"] = d.normal(T, (Hq + 2 * Hk) * D)
    s["q_in"], s["k_in"], s["v_in"] = s["qkv"].split([Hq * D, Hk * D, Hk * D], dim=1)
    s["wq"] = s["wk"] = None
    if case["norm"]:
        s["wq"], s["wk"] = ((1 + 0.1 * d.normal(D, dtype=F32)).to(BF16) for _ in range(2))
    s["max_position"] = max_position
    s["cos_sin"] = _angles(max_position, case["rot"], d.dev)
    s["q"] = d.zeros(T, Hq * D)


def _angles(n, rot, dev):
    """[n, rot]: the cosines of the rot/2 angles of every position, then their sines."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, dtype=F64, device=dev) / rot)
    a = torch.arange(n, dtype=F64, device=dev)[:, None] * f
    return torch.cat([a.cos(), a.sin()], dim=1).to(F32)


def _prepare_cache(d, case, s, filled):
    shape = (s["n_pages"], case["heads_kv"], case["page"], D)
    s["k_cache"], s["v_cache"] = (d.normal(*shape) if filled else d.zeros(*shape) for _ in range(2))


def _prepare_attention(d, case, s):
    T, Hq = s["T"], case["heads_q"]
    s["o"], s["lse"] = d.zeros(T, Hq * D), d.zeros(T, Hq, dtype=F32)
    if own:
        tl = s["lib"].tl
        sizes = tl.tl_paged_query(s["lib"].ctx, s["dims"])
        s["ws_bytes"] = sizes["ws_bytes"]
        s["schedule"], s["ws"] = d.zeros(sizes["schedule_bytes"] // 4, dtype=I32), d.zeros(s["ws_bytes"] // 4, dtype=I32)


def prepare(case, seed):
    d, op = _Draw(seed), case["op"]
    s = {"case": case}
    if own:
        s["lib"] = _Context()
    if op in ("norm_rope", "norm_rope_cache"):
        T = s["T"] = case["T"]
        s["new"], s["max_blocks"] = [T], 1
        _prepare_rows(d, case, s, T, max(2 * T, 4096))
        s["positions"] = torch.randint(0, s["max_position"], (T,), generator=d.g, device=d.dev, dtype=I32)
        if op == "norm_rope":
            s["k"] = d.zeros(T, case["heads_kv"] * D)
        else:
            s["n_pages"] = _pages(T, case["page"]) + 2
            s["slots"] = torch.randperm(s["n_pages"] * case["page"], generator=d.g, device=d.dev)[:T].to(I32)
            _prepare_cache(d, case, s, filled=False)
    else:
        _prepare_requests(d, case, s)
    if op in ("slots", "step"):
        _prepare_slots(d, case, s)
    if op == "step":
        _prepare_rows(d, case, s, s["T"], max(c + n for c, n in zip(s["ctx"], s["new"])))
    if op == "attention":
        s["q"] = d.normal(s["T"], case["heads_q"] * D)
        s["query_start"] = d.ints([0] + s["new"]).cumsum(0).to(I32)
        s["seq_lens"] = d.ints([c + n for c, n in zip(s["ctx"], s["new"])])
    if op in ("attention", "step"):
        _prepare_cache(d, case, s, filled=True)
    if own and op != "norm_rope":
        s["dims"] = s["lib"].tl.tl_paged_dims(batch=case.get("B", 1), max_tokens=s["T"], max_new=max(s["new"]), max_blocks=s["max_blocks"], page_size=case["page"],
                                              n_pages=s["n_pages"], heads_q=case.get("heads_q", 1), heads_kv=case.get("heads_kv", 1), head_dim=D,
                                              window=case.get("window", 0))
    if op in ("attention", "step"):
        _prepare_attention(d, case, s)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# One pass: the library's calls
# ---------------------------------------------------------------------------------------------------------------------
def _own_slots(s, stream):
    tl = s["lib"].tl
    tl.tl_paged_slots(s["lib"].ctx, s["dims"], s["ctx_lens"], s["new_lens"], s["free"], s["free"].numel(), s["free_from"], s["free_to"], s["table"],
                      s["query_start"], s["seq_lens"], s["slots"], s["positions"], s["counts"], stream)


def _own_rows(s, stream):
    c, tl = s["case"], s["lib"].tl
    row, Hq, Hk = s["qkv"].stride(0), c["heads_q"], c["heads_kv"]
    rotation = (s["positions"], s["cos_sin"], s["max_position"], c["rot"], c["pairs"] == "neighbours", stream)
    if c["op"] == "norm_rope":
        tl.tl_qk_norm_rope(s["lib"].ctx, s["q_in"], row, s["k_in"], row, s["q"], Hq * D, s["k"], Hk * D, s["T"], Hq, Hk, D, s["wq"], s["wk"], EPS, *rotation)
    else:
        tl.tl_qk_norm_rope_cache(s["lib"].ctx, s["dims"], s["q_in"], row, s["k_in"], row, s["v_in"], row, s["q"], Hq * D, s["k_cache"], s["v_cache"], s["slots"],
                                 s["wq"], s["wk"], EPS, *rotation)


def _own_attention(s, stream):
    tl, row = s["lib"].tl, s["case"]["heads_q"] * D
    tl.tl_paged_schedule(s["lib"].ctx, s["dims"], s["query_start"], s["seq_lens"], s["schedule"], s["schedule"].numel() * 4, stream)
    tl.tl_paged_attention(s["lib"].ctx, s["dims"], s["q"], row, s["k_cache"], s["v_cache"], s["table"], s["schedule"], s["o"], row, s["lse"], SCALE, s["ws"],
                          s["ws_bytes"], stream)


# ---------------------------------------------------------------------------------------------------------------------
# One pass: the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _plain_slots(s):
    P, T, width, free = s["case"]["page"], s["T"], s["max_blocks"], s["free"].long()
    ctx, new = s["ctx_lens"].long(), s["new_lens"].long()
    new = torch.minimum(new.clamp(min=0), width * P - ctx)
    end = new.cumsum(0).clamp(max=T)
    start = torch.cat([end.new_zeros(1), end])
    n = start[1:] - start[:-1]
    seq = ctx + n
    have, want = (ctx + P - 1) // P, (seq + P - 1) // P
    first = s["free_from"].long() + (want - have).cumsum(0) - (want - have)       # place of a request's first new page in the free list

    def from_list(i):
        return torch.where(i < free.numel(), free[i.clamp(0, free.numel() - 1)], -1)

    j = torch.arange(width, device=ctx.device)
    fresh = (j >= have[:, None]) & (j < want[:, None])
    s["table"].copy_(torch.where(fresh, from_list(first[:, None] + j - have[:, None]), s["table"].long()))
    t = torch.arange(T, device=ctx.device)
    b = torch.searchsorted(end, t, right=True).clamp(max=len(ctx) - 1)
    real = t < end[-1]
    pos = ctx[b] + t - start[b]
    page = s["table"].long()[b, (pos // P).clamp(0, width - 1)]
    s["slots"].copy_(torch.where(real & (page >= 0), page * P + pos % P, -1))
    s["positions"].copy_(torch.where(real, pos, 0))
    s["query_start"].copy_(start)
    s["seq_lens"].copy_(seq)
    taken = torch.minimum((want - have).sum(), free.numel() - s["free_from"][0])
    s["free_to"].copy_(s["free_from"] + taken)
    s["counts"].copy_(torch.stack([end[-1], taken, (want - have).sum() - taken, s["new_lens"].clamp(min=0).sum() - end[-1]]))


def _normed_rotated(x, heads, w, cos, sin, neighbours, dtype=F32):
    """[T, heads*D] -> [T, heads, D], unrounded."""
    x = x.to(dtype).reshape(x.shape[0], heads, D)
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.to(dtype)
    half = cos.shape[-1]
    cos, sin = cos[:, None].to(dtype), sin[:, None].to(dtype)
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    if neighbours:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = r[..., :half], r[..., half:]
        r = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([r, rest], dim=-1)


def _plain_rows(s):
    c = s["case"]
    cs = s["cos_sin"][s["positions"].long()]
    half = c["rot"] // 2
    q, k = (_normed_rotated(x, h, w, cs[:, :half], cs[:, half:], c["pairs"] == "neighbours").to(BF16)
            for x, h, w in ((s["q_in"], c["heads_q"], s["wq"]), (s["k_in"], c["heads_kv"], s["wk"])))
    s["q"].copy_(q.flatten(1))
    if c["op"] == "norm_rope":
        s["k"].copy_(k.flatten(1))
    else:
        page, at = s["slots"].long() // c["page"], s["slots"].long() % c["page"]
        s["k_cache"][page, :, at] = k
        s["v_cache"][page, :, at] = s["v_in"].reshape(s["T"], -1, D)


def _attended(q, k, v, ctx, window, dtype):
    """q [n, G, D] of one key head at positions ctx.., k and v [ctx + n, D] -> o [n, G, D], lse [n, G]."""
    n, G, _ = q.shape
    at = torch.arange(ctx, ctx + n, device=q.device)[:, None, None]
    key = torch.arange(ctx + n, device=q.device)
    seen = key <= at
    if window:
        seen = seen & (key > at - window)
    x = torch.matmul(q.to(dtype).reshape(n * G, D), k.to(dtype).t()).reshape(n, G, -1) * SCALE
    x = x.masked_fill(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - m)
    l = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(n * G, -1), v.to(dtype)).reshape(n, G, D) / l
    return o, (m + torch.log(l)).squeeze(-1)


def _attention_of(s, q, dtype):
    """Request by request, key head by key head; yields (rows, query heads, o, lse)."""
    c, row = s["case"], 0
    Hk, P = c["heads_kv"], c["page"]
    G = c["heads_q"] // Hk
    for b, (ctx, n) in enumerate(zip(s["ctx"], s["new"])):
        pages = s["table"][b, :_pages(ctx + n, P)].long()
        lo = max(0, ctx - c["window"] + 1) // P if c["window"] else 0       # no query of the request sees an earlier page
        k, v = (x[pages[lo:]].transpose(0, 1).reshape(Hk, -1, D)[:, :ctx + n - lo * P] for x in (s["k_cache"], s["v_cache"]))
        rows = slice(row, row + n)
        qb = q[rows].reshape(n, c["heads_q"], D)
        for h in range(Hk):
            heads = slice(h * G, (h + 1) * G)
            yield (rows, heads) + _attended(qb[:, heads], k[h], v[h], ctx - lo * P, c["window"], dtype)
        row += n


def _plain_attention(s):
    o = s["o"].reshape(s["T"], -1, D)
    for rows, heads, oh, lse in _attention_of(s, s["q"], F32):
        o[rows, heads] = oh.to(BF16)
        s["lse"][rows, heads] = lse


def run(s):
    op = s["case"]["op"]
    if own:
        stream = torch.cuda.current_stream()
        slots, rows, attention = (lambda f=f: f(s, stream) for f in (_own_slots, _own_rows, _own_attention))
    else:
        slots, rows, attention = (lambda f=f: f(s) for f in (_plain_slots, _plain_rows, _plain_attention))
    out = {}
    if op in ("slots", "step"):
        slots()
        out.update((x, s[x]) for x in ("table", "query_start", "seq_lens", "slots", "positions", "free_to", "counts"))
    if op in ("norm_rope", "norm_rope_cache", "step"):
        rows()
        out.update((x, s[x]) for x in (("q", "k") if op == "norm_rope" else ("q", "k_cache", "v_cache")))
    if op in ("attention", "step"):
        attention()
        out.update((x, s[x]) for x in ("o", "lse"))
    return out


# ---------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------------
def _exact_rows(x, heads, w, pos, rot, neighbours, cos_sin):
    """Every rotated pair as a complex number times exp(i angle), the angle's cosine and sine taken from the given table."""
    T = x.shape[0]
    x = x.double().reshape(T, heads, D)
    if w is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * w.double()
    turn = torch.complex(*(cos_sin.double()[pos.long()][:, None, i * rot // 2:(i + 1) * rot // 2].contiguous() for i in (0, 1)))
    first = torch.arange(0, rot, 2, device=x.device) if neighbours else torch.arange(rot // 2, device=x.device)
    second = first + (1 if neighbours else rot // 2)
    z = torch.complex(x[..., first], x[..., second]) * turn
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_attention(s, c, q, k_cache, v_cache, table, o, lse):
    """Key by key of the flat cache: the slots a request sees, one key head at a time."""
    P, Hk = c["page"], c["heads_kv"]
    G, row = c["heads_q"] // Hk, 0
    for b, (ctx, n) in enumerate(zip(s["ctx"], s["new"])):
        key = torch.arange(ctx + n, device=q.device)
        slot = table[b, key // P].long() * P + key % P
        age = torch.arange(ctx, ctx + n, device=q.device)[:, None] - key[None]            # how far the key lies behind the query
        hidden = (age < 0) | (age >= (c["window"] or ctx + n))
        for h in range(Hk):
            kh, vh = (x[slot // P, h, slot % P].double() for x in (k_cache, v_cache))
            for g in range(h * G, (h + 1) * G):
                x = (q[row:row + n, g].double() @ kh.t()) * SCALE
                x[hidden] = -math.inf
                z = torch.logsumexp(x, dim=-1)
                o[row:row + n, g] = torch.exp_(x.sub_(z[:, None])) @ vh
                lse[row:row + n, g] = z
        row += n


def exact(case, seed):
    op = case["op"]
    if op == "slots":
        return None                     # whole numbers
    s = prepare(case, seed)
    out = {}
    if op == "step":
        with torch.no_grad():
            _plain_slots(s)             # whole numbers, which the rest is laid out by
        out.update((x, None) for x in ("table", "query_start", "seq_lens", "slots", "positions", "free_to", "counts"))
    q = s["q"]
    kc, vc = s.get("k_cache"), s.get("v_cache")
    if op != "attention":
        q, k = (_exact_rows(s[x], h, w, s["positions"], case["rot"], case["pairs"] == "neighbours", s["cos_sin"])
                for x, h, w in (("q_in", case["heads_q"], s["wq"]), ("k_in", case["heads_kv"], s["wk"])))
        out["q"] = q.flatten(1)
        if op == "norm_rope":
            out["k"] = k.flatten(1)
        else:
            kc, vc = kc.double(), vc.double()
            for x, y in ((kc, k), (vc, s["v_in"].reshape(s["T"], -1, D).double())):
                x[s["slots"].long() // case["page"], :, s["slots"].long() % case["page"]] = y
            out["k_cache"], out["v_cache"] = kc, vc
    if op in ("attention", "step"):
        if op == "step":                # the attention reads what the cache and the query rows hold: rounded values
            q, kc = q.to(BF16), kc.to(BF16)
        T, Hq = s["T"], case["heads_q"]
        out["o"] = torch.zeros(T, Hq, D, dtype=F64, device=q.device)
        out["lse"] = torch.zeros(T, Hq, dtype=F64, device=q.device)
        _exact_attention(s, case, q.reshape(T, Hq, D), kc, vc, s["table"], out["o"], out["lse"])
        out["o"] = out["o"].flatten(1)
        if op == "step":                # a query or key that lies next to a rounding border moves the logarithm by more than 32 bits show
            out["lse"] = None
    return out


# ---------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------------
def _work_slots(case):
    ctx, new = _lengths(case)
    P, T = case["page"], sum(new)
    fresh = sum(_pages(c + n, P) - _pages(c, P) for c, n in zip(ctx, new))
    cut = sum(c % P > 0 for c in ctx)               # pages that are partly filled: their entry of the table is read
    return 4.0 * (2 * len(new) + fresh + cut + fresh + 2 * T + 2 * len(new) + 1), 0.0


def _work_rows(case, T):
    Hq, Hk = case["heads_q"], case["heads_kv"]
    moved = Hq + Hk * (1 if case["op"] == "norm_rope" else 2)
    return 2.0 * 2 * T * moved * D + 4.0 * T * (case["rot"] + 2), 8.0 * T * (Hq + Hk) * D


def _work_attention(case):
    ctx, new = _lengths(case)
    w, Hq, Hk = case["window"], case["heads_q"], case["heads_kv"]
    pairs = keys = 0
    for c, n in zip(ctx, new):
        keys += c + n - (max(0, c - w + 1) if w else 0)
        whole = n * c + n * (n + 1) // 2                                          # every earlier token
        m = c + n - w                                                             # without the pairs further apart than the window
        cut = (m * (m + 1) - max(0, m - n) * (max(0, m - n) + 1)) // 2 if w and m > 0 else 0
        pairs += whole - cut
    return 2.0 * 2 * keys * Hk * D + sum(new) * Hq * (4.0 * D + 4), 4.0 * D * Hq * pairs


def work(case):
    op, b, f = case["op"], 0.0, 0.0
    parts = []
    if op in ("slots", "step"):
        parts.append(_work_slots(case))
    if op in ("norm_rope", "norm_rope_cache"):
        parts.append(_work_rows(case, case["T"]))
    if op == "step":
        parts.append(_work_rows(case, sum(_lengths(case)[1])))
    if op in ("attention", "step"):
        parts.append(_work_attention(case))
    for x, y in parts:
        b, f = b + x, f + y
    return {"bytes": b, "flops": f}
