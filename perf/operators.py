"""Serving from a paged cache: the work of its operators as cases that can be timed and checked.

Kinds of case, each one pass through an entry point of `paper_2608_20172_amd.binding`:
  map     relation_page_map: block tables, slots and positions of a step from request lengths
  append  relation_paged_append: RoPE on q and k, Givens mixing of v, rows written to their slots
  decode  relation_paged_decode: Full Relation of one new token per request over the cache's pages
  sample  relation_sample: temperature, top-k, top-p and min-p from given random numbers

`run` computes the plain form in 32 bits from elementary torch operations, or, where `own` is true,
calls the framework. `exact` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TAU = 2.0
ROPE_BASE = 1.0e4
TINY = 2.0 ** -126  # random numbers count as at least this
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One user, a short answer, the 30M model's 8 heads of width 64: launches and host time count.
        {"name": "decode_one", "kind": "decode", "B": 1, "H": 8, "G": 1, "T": 201, "low": 1.0, "D": 64, "page": 16,
         "dtype": "bf16", "layout": "hnd"},
        # A batch of requests of mixed lengths at the 100M-scale layer.
        {"name": "decode_batch", "kind": "decode", "B": 64, "H": 12, "G": 1, "T": 4096, "low": 0.25, "D": 64,
         "page": 16, "dtype": "bf16", "layout": "hnd"},
        # Two users with very long contexts, the widest head: the largest reads.
        {"name": "decode_long", "kind": "decode", "B": 2, "H": 16, "G": 1, "T": 65536, "low": 0.9, "D": 128,
         "page": 64, "dtype": "bf16", "layout": "nhd"},
        # Key and value heads shared by four query heads each.
        {"name": "decode_shared", "kind": "decode", "B": 32, "H": 4, "G": 4, "T": 8192, "low": 0.1, "D": 128,
         "page": 32, "dtype": "bf16", "layout": "nhd"},
        # The paper's width 80 in 32 bits, an odd batch.
        {"name": "decode_f32", "kind": "decode", "B": 7, "H": 8, "G": 1, "T": 2047, "low": 0.02, "D": 80, "page": 16,
         "dtype": "f32", "layout": "hnd"},
        # A decode step of 64 requests: one token each, a new page for one in sixteen.
        {"name": "map_step", "kind": "map", "B": 64, "added": 1, "T": 4096, "page": 16},
        # A batch of prompts taken in, with requests that go on.
        {"name": "map_prompts", "kind": "map", "B": 96, "added": 2048, "T": 4096, "page": 16},
        # The rows of a decode step, 64 requests, 8 heads of width 80.
        {"name": "append_step", "kind": "append", "B": 64, "N": 64, "H": 8, "G": 1, "D": 80, "Dc": 80, "page": 16,
         "dtype": "bf16", "pairing": "A", "layout": "hnd"},
        # The rows of prompts, 12 heads of width 64.
        {"name": "append_prompts", "kind": "append", "B": 9, "N": 16384, "H": 12, "G": 1, "D": 64, "Dc": 64,
         "page": 16, "dtype": "bf16", "pairing": "B", "layout": "nhd"},
        # One user's next token from a vocabulary of 32000, in 32 bits.
        {"name": "sample_one", "kind": "sample", "B": 1, "V": 32000, "dtype": "f32", "slope": 1.2, "rows": "all",
         "order": "mixed"},
        # A batch, every filter on, rows not on 16-byte boundaries.
        {"name": "sample_batch", "kind": "sample", "B": 64, "V": 50257, "dtype": "bf16", "slope": 1.1, "rows": "all",
         "order": "ranked"},
        # A large batch and vocabulary: rows without filters, with top-p alone, with all of them and greedy ones.
        {"name": "sample_large", "kind": "sample", "B": 256, "V": 131072, "dtype": "f32", "slope": 1.2,
         "rows": "each", "order": "mixed"},
    ]


# ---------------------------------------------------------------------------
# Drawn cases: the same kinds over their ranges
# ---------------------------------------------------------------------------
def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(max(hi, lo))))


def _int(rng, lo, hi):
    return max(lo, min(hi, int(round(_log(rng, lo, hi)))))


def draw(rng):
    kind = rng.choice(["decode", "decode", "decode", "sample", "sample", "append", "append", "map"])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    layout = rng.choice(["hnd", "nhd"])
    page = rng.choice([8, 16, 16, 32, 64, 128])
    if kind == "decode":
        D = rng.choice([32, 48, 64, 64, 80, 96, 128])
        H, G = rng.choice([1, 2, 4, 8, 12, 16]), rng.choice([1, 1, 1, 2, 3, 4, 8])
        T = _int(rng, 1, 65536)
        most = (1 << 27) // (2 if dtype == "f32" else 1)
        B = _int(rng, 1, min(256, max(1, most // (H * T * D))))
        return {"kind": kind, "B": B, "H": H, "G": G, "T": T, "low": rng.uniform(0.01, 1.0), "D": D, "page": page,
                "dtype": dtype, "layout": layout}
    if kind == "sample":
        B = _int(rng, 1, 256)
        V = _int(rng, 1000, min(131072, (1 << 25) // B))
        return {"kind": kind, "B": B, "V": V, "dtype": dtype, "slope": rng.uniform(1.0, 1.6),
                "rows": rng.choice(["all", "each"]), "order": rng.choice(["mixed", "ranked"])}
    if kind == "append":
        D = rng.choice([48, 60, 64, 80, 128])
        B = _int(rng, 1, 64)
        return {"kind": kind, "B": B, "N": _int(rng, B, 16384 if dtype == "bf16" else 8192), "H": rng.choice([2, 4, 8, 12]),
                "G": rng.choice([1, 1, 2, 4]) if D <= 64 else 1, "D": D, "Dc": (D + 15) // 16 * 16, "page": page,
                "dtype": dtype, "pairing": rng.choice(["A", "B"]), "layout": layout}
    return {"kind": kind, "B": _int(rng, 1, 1024), "added": _int(rng, 1, 1024), "T": _int(rng, 64, 4096), "page": page}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _spread(n, lo, hi, g, dev):
    """n whole numbers spread evenly from lo to hi, in an order of the seed (so their sum is the case's own)."""
    x = torch.linspace(lo, hi, n, device=dev, dtype=torch.float64) if n > 1 else torch.full((1,), float(hi), device=dev)
    return x.round().to(torch.int32)[torch.randperm(n, device=dev, generator=g)]


def _table(lens, page, g, dev):
    """Block tables of requests that hold lens[b] tokens: pages in a random order, -1 past the last; and the pool's
    pages, as many as so many tokens of so many requests can take."""
    used = (lens.long() + page - 1) // page
    W, pool = int(used.max()), (int(lens.sum()) + lens.numel() * (page - 1)) // page + 3
    ids = torch.randperm(pool, device=dev, generator=g)
    col = torch.arange(W, device=dev)[None]
    at = (used.cumsum(0) - used)[:, None] + col
    return torch.where(col < used[:, None], ids[at.clamp(max=pool - 1)], -1).to(torch.int32), pool


def _cache(c, pages, width, g, dev):
    shape = (pages, c["page"], c["H"], width) if c["layout"] == "nhd" else (pages, c["H"], c["page"], width)
    x = torch.randn(shape, device=dev, generator=g, dtype=torch.float32).to(DTYPES[c["dtype"]])
    return x.transpose(1, 2) if c["layout"] == "nhd" else x


def _lengths64(c):
    """The decode case's lengths, unordered."""
    lo, hi = max(1.0, round(c["low"] * c["T"])), float(c["T"])
    return [hi] if c["B"] == 1 else [round(lo + i * (hi - lo) / (c["B"] - 1)) for i in range(c["B"])]


def prepare(c, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    s = {"case": c}
    B = c["B"]
    if c["kind"] == "map":
        page = c["page"]
        s["cached"] = _spread(B, 0, c["T"], g, dev)
        added = torch.ones(B, dtype=torch.int32, device=dev)
        added[B // 3:] = _spread(B - B // 3, 1, c["added"], g, dev)  # a third of the requests add one token
        s["added"] = added[torch.randperm(B, device=dev, generator=g)]
        new = s["cached"].long() + s["added"].long()
        width = (c["T"] + c["added"] + page - 1) // page
        have = (s["cached"].long() + page - 1) // page
        need = (new + page - 1) // page - have
        n_have, n_need = int(have.sum()), int(need.sum())
        ids = torch.randperm(n_have + n_need + 8, device=dev, generator=g).to(torch.int32)
        col = torch.arange(width, device=dev)[None]
        at = (have.cumsum(0) - have)[:, None] + col
        s["table"] = torch.where(col < have[:, None], ids[at.clamp(max=max(n_have - 1, 0))], -1).to(torch.int32)
        s["free"] = ids[n_have:].contiguous()
        s["tokens"] = int(s["added"].sum()) + 5  # the step's token buffers hold a few more
        return s
    if c["kind"] == "sample":
        V = c["V"]
        rank = torch.rand(B, V, device=dev, generator=g) * V if c["order"] == "mixed" else \
            torch.arange(V, device=dev, dtype=torch.float32).expand(B, V)
        x = -c["slope"] * torch.log1p(rank) + 0.3 * torch.randn(B, V, device=dev, generator=g)
        s["logits"] = x.to(DTYPES[c["dtype"]])
        s["noise"] = torch.empty(B, V, device=dev).exponential_(generator=g)
        s["temperature"] = 0.6 + 0.6 * torch.rand(B, device=dev, generator=g)
        s["top_k"] = torch.randint(20, 80, (B,), device=dev, generator=g, dtype=torch.int32)
        s["top_p"] = 0.85 + 0.13 * torch.rand(B, device=dev, generator=g)
        s["min_p"] = 0.02 * torch.rand(B, device=dev, generator=g)
        if c["rows"] == "each":  # row b: no filter, top-p alone, all filters, greedy
            kind = torch.arange(B, device=dev) % 4
            s["top_k"][(kind < 2)] = 0
            s["top_p"][kind == 0] = 1.0
            s["min_p"][kind < 2] = 0.0
            s["temperature"][kind == 3] = 0.0
        return s
    page, t = c["page"], DTYPES[c["dtype"]]
    Hq = c["H"] * c["G"]
    if c["kind"] == "append":
        N, D = c["N"], c["D"]
        first = _spread(B, 0, 2000, g, dev).long()
        many = torch.full((B,), max(1, N // (2 * B)), device=dev)
        many[0] += N - int(many.sum())  # one prompt takes half of the tokens
        table, pages = _table((first + many).to(torch.int32), page, g, dev)
        req = torch.repeat_interleave(torch.arange(B, device=dev), many, output_size=N)
        pos = first[req] + torch.arange(N, device=dev) - (many.cumsum(0) - many)[req]
        s["slots"] = table.long()[req, pos // page] * page + pos % page
        s["positions"] = pos.to(torch.int32)
        for n, h in (("q", Hq), ("k", c["H"]), ("v", c["H"])):
            s[n] = torch.randn(N, h, D, device=dev, generator=g).to(t)
        s["theta"] = (torch.rand(c["H"] // 2, device=dev, generator=g) * 2 - 1) * math.pi
        s["k_cache"], s["v_cache"] = _cache(c, pages, c["Dc"], g, dev), _cache(c, pages, c["Dc"], g, dev)
        return s
    lens = torch.tensor(_lengths64(c), device=dev).to(torch.int32)[torch.randperm(B, device=dev, generator=g)]
    s["lengths"] = lens
    s["table"], pages = _table(lens, page, g, dev)
    s["k_cache"], s["v_cache"] = _cache(c, pages, c["D"], g, dev), _cache(c, pages, c["D"], g, dev)
    used = torch.zeros(pages, page, dtype=torch.bool, device=dev)
    at = torch.arange(s["table"].shape[1] * page, device=dev)
    slot = s["table"].long().repeat_interleave(page, 1) * page + at % page
    used.view(-1)[slot[at[None] < lens[:, None]]] = True
    for x in (s["k_cache"], s["v_cache"]):  # what no request holds is whatever was there before
        x.masked_fill_(~used[:, None, :, None], math.nan)
    s["q"] = torch.randn(B, Hq, c["D"], device=dev, generator=g).to(t)
    s["lam"] = torch.full((1,), 0.5, device=dev)  # the paper's initial value
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"map": _map, "append": _append, "decode": _decode, "sample": _sample}[kind](s)
    from paper_2608_20172_amd import binding as R
    if kind == "map":
        return R.relation_page_map(s["cached"], s["added"], s["table"], s["free"], s["case"]["page"], s["tokens"])
    if kind == "append":
        q = R.relation_paged_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["slots"], s["positions"], q=s["q"],
                                    theta=s["theta"], pairing=s["case"]["pairing"], rope_base=ROPE_BASE)
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if kind == "decode":
        return R.relation_paged_decode(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["lam"])
    return R.relation_sample(s["logits"], s["noise"], temperature=s["temperature"], top_k=s["top_k"],
                             top_p=s["top_p"], min_p=s["min_p"])


def _map(s):
    cached, added, free, page, N = s["cached"].long(), s["added"].long(), s["free"], s["case"]["page"], s["tokens"]
    B, W = s["table"].shape
    have, want = (cached + page - 1) // page, (cached + added + page - 1) // page
    valid = (cached >= 0) & (added >= 0) & (want <= W)
    need = torch.where(valid, want - have, 0)
    tokens = added.clamp(min=0)
    end = tokens.cumsum(0)
    taken = need.cumsum(0)
    served = valid & ((tokens == 0) | (end <= N)) & ((need == 0) | (taken <= free.numel()))
    col = torch.arange(W, device=free.device)[None]
    fresh = served[:, None] & (col >= have[:, None]) & (col < want[:, None])
    src = (taken - need)[:, None] + col - have[:, None]
    s["table"].copy_(torch.where(fresh, free[src.clamp(0, max(free.numel() - 1, 0))], s["table"]))
    n = torch.arange(N, device=free.device)
    b = (n[:, None] >= end[None]).sum(1)
    inside = b < B
    b = b.clamp(max=B - 1)
    inside = inside & served[b]
    pos = cached[b] + n - (end - tokens)[b]
    slot = s["table"].long()[b, (pos // page).clamp(0, W - 1)] * page + pos % page
    start = torch.cat([end.new_zeros(1), end]).clamp(max=N)
    return {"table": s["table"], "lengths": torch.where(served, cached + added, 0).to(torch.int32),
            "row_start": start.to(torch.int32), "slots": torch.where(inside, slot, -1),
            "positions": torch.where(inside, pos, -1).to(torch.int32),
            "counts": torch.stack([torch.where(served, need, 0).sum(), torch.where(served, tokens, 0).sum(),
                                   (~served).sum()]).to(torch.int32)}


def _rotate(x, cs, sn):
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * cs - b * sn, a * sn + b * cs], -1)


def _pairs(H, pairing, dev):
    first = torch.arange(0, H, 2, device=dev) + (0 if pairing == "A" else 1)
    return first, (first + 1) % H


def _append(s):
    c = s["case"]
    D, Dc, page = c["D"], c["Dc"], c["page"]
    # the angle in 64 bits: a position times a frequency leaves nothing of 32 bits' fraction in a long context
    j = torch.arange(D // 2, dtype=torch.float64, device=s["k"].device)
    ang = s["positions"].double()[:, None] * ROPE_BASE ** (-2.0 * j / D)
    cs, sn = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    q, k = _rotate(s["q"].float(), cs, sn), _rotate(s["k"].float(), cs, sn)
    first, second = _pairs(c["H"], c["pairing"], q.device)
    ct, st = torch.cos(s["theta"])[None, :, None], torch.sin(s["theta"])[None, :, None]
    v = s["v"].float()
    a, b = v[:, first], v[:, second]
    mixed = torch.empty_like(v)
    mixed[:, first] = ct * a - st * b
    mixed[:, second] = st * a + ct * b
    pad = torch.nn.functional.pad
    at, row = s["slots"] // page, s["slots"] % page
    t = s["k"].dtype
    s["k_cache"][at, :, row] = pad(k, (0, Dc - D)).to(t)
    s["v_cache"][at, :, row] = pad(mixed, (0, Dc - D)).to(t)
    return {"q": pad(q, (0, Dc - D)).to(t), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _gathered(x, table, n):
    """[B, H, W page, D] of the pages of each request, zero past its length, in 32 bits."""
    B, W = table.shape
    y = x[table.clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(B, x.shape[1], W * x.shape[2], x.shape[3]).float()
    return y.masked_fill_(torch.arange(y.shape[2], device=y.device)[None, None, :, None] >= n[:, None, None, None], 0.0)


def _decode(s):
    c = s["case"]
    B, H, G, D = c["B"], c["H"], c["G"], c["D"]
    n = s["lengths"].long()
    K, V = _gathered(s["k_cache"], s["table"], n), _gathered(s["v_cache"], s["table"], n)
    q = s["q"].float().view(B, H, G, D) / math.sqrt(D)
    U = (K @ q.transpose(2, 3).contiguous()).transpose(2, 3)  # [B, H, G, T]
    j = torch.arange(K.shape[2], device=K.device)[None, None, None]
    last = (n - 1)[:, None, None, None]
    E = (U * torch.sigmoid(U)).masked_fill(j >= last, -math.inf)
    S = torch.sigmoid(torch.gather(U, 3, last.expand(B, H, G, 1)) / TAU)
    m = E.amax(3, keepdim=True)
    P = torch.exp(E - m.clamp(min=-3.0e38))
    l = P.sum(3, keepdim=True)
    ln = torch.log(n.float())[:, None, None, None]
    A = torch.log(l) + m - s["lam"] * ln
    vi = torch.gather(V, 2, last.expand(B, H, 1, D))
    z = (P.contiguous() @ V) / l.clamp(min=1.0e-30)
    y = torch.sigmoid(S - A) * vi + torch.sigmoid(A - S) * z
    top = torch.maximum(S, A)
    M = top + torch.log(torch.exp(S - top) + torch.exp(A - top)) + s["lam"] * ln
    return {"o": y.reshape(B, H * G, D).to(s["q"].dtype), "row_stat": M.reshape(B, H * G)}


def _sample(s):
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), -math.inf, x)
    B, V = x.shape
    greedy = s["temperature"] == 0
    T = torch.where(greedy, 1.0, s["temperature"])[:, None]
    k = torch.where(greedy, 1, torch.where(s["top_k"] <= 0, V, s["top_k"].long()))[:, None]
    v, at = torch.sort(x, dim=1, descending=True, stable=True)  # ties: lower index first
    d = torch.where(v == v[:, :1], 0.0, (v - v[:, :1]) / T)
    w = torch.exp(d)
    Z = w.sum(1, keepdim=True)
    before = w.cumsum(1) - w
    rank = torch.arange(V, device=x.device)[None]
    top_p = s["top_p"][:, None]
    keep = (rank < k) & ((before < top_p * Z) | (top_p >= 1)) & (w >= s["min_p"][:, None])
    keep[:, 0] = True
    score = torch.where(keep, w / s["noise"].gather(1, at).clamp(min=TINY), -1.0)
    best = score == score.amax(1, keepdim=True)
    token = torch.where(best, at, V).amin(1)
    place = torch.argmax((at == token[:, None]).to(torch.uint8), 1, keepdim=True)
    logprob = (d.gather(1, place) - torch.log(Z))[:, 0]
    none = v[:, 0] == -math.inf
    return {"tokens": torch.where(none, -1, token), "logprob": torch.where(none, math.nan, logprob)}


# ---------------------------------------------------------------------------
# The work that a pass cannot do without
# ---------------------------------------------------------------------------
def work(c):
    B = c["B"]
    if c["kind"] == "map":
        added = B // 3 + (B - B // 3) * (c["added"] if B - B // 3 == 1 else (1 + c["added"]) / 2.0)
        pages = added / c["page"]
        # lengths and pages taken in; slots and positions of the tokens, pages, lengths and starts out
        return {"bytes": 8 * B + 4 * pages + 12 * added + 4 * pages + 8 * B, "flops": 8.0 * (added + B)}
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "append":
        rows = c["N"] * c["H"] * (c["G"] + 2)
        return {"bytes": rows * (c["D"] + c["Dc"]) * es + 12 * c["N"], "flops": 3.0 * rows * c["D"]}
    if c["kind"] == "decode":
        keys = sum(_lengths64(c))
        Hq = c["H"] * c["G"]
        # K and V rows of every entry and the page ids; q in, o and row_stat out
        return {"bytes": 2 * c["H"] * keys * c["D"] * es + 4 * keys / c["page"] + 2 * B * Hq * c["D"] * es + 4 * B * Hq,
                "flops": 4.0 * Hq * keys * c["D"]}
    # the logits, and the random numbers of the rows without a filter
    free = (B + 3) // 4 if c["rows"] == "each" else 0
    return {"bytes": B * c["V"] * es + 4.0 * free * c["V"] + 28 * B, "flops": 4.0 * B * c["V"]}


# ---------------------------------------------------------------------------
# The same outputs in 64 bits
# ---------------------------------------------------------------------------
def exact(c, seed):
    if c["kind"] == "map":
        return None  # whole numbers alone
    s = prepare(c, seed)
    f = torch.float64
    if c["kind"] == "append":
        page, D, Dc = c["page"], c["D"], c["Dc"]
        w = ROPE_BASE ** (-torch.arange(0, D, 2, device=s["k"].device, dtype=f) / D)
        turn = torch.polar(torch.ones_like(w), w)[None] ** s["positions"][:, None]  # e^(i t w)
        half = D // 2
        out = {}
        for n in ("q", "k"):
            z = torch.complex(s[n][..., :half].to(f), s[n][..., half:].to(f)) * turn[:, None]
            out[n] = torch.cat([z.real, z.imag, z.real.new_zeros(*z.shape[:2], Dc - D)], -1)
        v = s["v"].to(f)
        mixed = torch.zeros(*v.shape[:2], Dc, dtype=f, device=v.device)
        first, second = _pairs(c["H"], c["pairing"], v.device)
        for th, a, b in zip(s["theta"].to(f), first.tolist(), second.tolist()):
            mixed[:, a, :D] = torch.cos(th) * v[:, a] - torch.sin(th) * v[:, b]
            mixed[:, b, :D] = torch.sin(th) * v[:, a] + torch.cos(th) * v[:, b]
        res = {"q": out["q"]}
        for n, rows in (("k_cache", out["k"]), ("v_cache", mixed)):
            res[n] = s[n].to(f)
            res[n][s["slots"] // page, :, s["slots"] % page] = rows
        return res
    if c["kind"] == "decode":
        G, page, D = c["G"], c["page"], c["D"]
        o = torch.empty(s["q"].shape, dtype=f, device=s["q"].device)
        M = torch.empty(s["q"].shape[:2], dtype=f, device=s["q"].device)
        lam = s["lam"][0].to(f)
        for b, n in enumerate(s["lengths"].tolist()):
            ids = s["table"][b, : (n + page - 1) // page].long()
            for h in range(c["H"]):
                k, v = (s[x][ids, h].reshape(-1, D)[:n].to(f) for x in ("k_cache", "v_cache"))
                for r in range(h * G, (h + 1) * G):
                    U = (k @ s["q"][b, r].to(f)) / math.sqrt(D)
                    R = U * torch.sigmoid(U) - lam * math.log(n)
                    R[-1] = torch.sigmoid(U[-1] / TAU)
                    lse = torch.logsumexp(R, 0)
                    o[b, r] = torch.exp(R - lse) @ v
                    M[b, r] = lse + lam * math.log(n)
        return {"o": o, "row_stat": M}
    lp = torch.empty(c["B"], dtype=f, device=s["logits"].device)
    for b in range(c["B"]):
        x = s["logits"][b].to(f)
        T, k, p, mp = (float(s[n][b]) for n in ("temperature", "top_k", "top_p", "min_p"))
        k, T = (1, 1.0) if T == 0 else (int(k) if k > 0 else c["V"], T)
        q = torch.softmax(x / T, 0)
        order = torch.argsort(x, descending=True, stable=True)
        qs = q[order]
        keep = (torch.arange(c["V"], device=x.device) < k) & (qs >= mp * qs[0])
        if p < 1:
            keep &= qs.cumsum(0) - qs < p
        keep[0] = True
        kept = order[keep]
        lp[b] = torch.log(q[kept[torch.argmax(q[kept] / s["noise"][b, kept].to(f))]])
    return {"tokens": None, "logprob": lp}
