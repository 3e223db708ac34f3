"""Prompts taken in by chunks: the work of their operators as cases that can be timed and checked.

Kinds of case, each one pass through entry points of `paper_2608_20172_amd.binding`:
  prefill   relation_paged_prefill: Full Relation of the new tokens of several requests over a paged cache
  norm      relation_qk_norm_fwd: RMS norm of each query and key head and the position rotation, in one pass
  normgrad  relation_qk_norm_bwd: its gradients, of both inputs and both weights
  score     relation_token_logprobs_fwd: log-probabilities of given tokens, entropy, rank and top alternatives
  train     relation_token_logprobs_fwd and _bwd: the first two and the gradient of a sum of them by the logits

`run` computes the plain form in 32 bits from elementary torch operations, or, where `own` is true,
calls the framework. `exact` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TAU = 2.0
ROPE_BASE = 1.0e4
EPS = 1.0e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One user's follow-up question of a few tokens after a short talk, the 30M model's 8 heads of width 64: latency.
        {"name": "prefill_one", "kind": "prefill", "B": 1, "H": 8, "G": 1, "D": 64, "cached": 201, "low": 1.0,
         "added": 24, "ones": 0.0, "page": 16, "dtype": "bf16", "layout": "hnd"},
        # A batch of fresh prompts of mixed lengths at the 100M-scale layer.
        {"name": "prefill_prompts", "kind": "prefill", "B": 8, "H": 12, "G": 1, "D": 64, "cached": 0, "low": 1.0,
         "added": 2048, "ones": 0.0, "page": 16, "dtype": "bf16", "layout": "nhd"},
        # One chunk of a very long prompt, key heads shared by four query heads each, the widest head.
        {"name": "prefill_long", "kind": "prefill", "B": 1, "H": 4, "G": 4, "D": 128, "cached": 32768, "low": 1.0,
         "added": 2048, "ones": 0.0, "page": 64, "dtype": "bf16", "layout": "nhd"},
        # A step that decodes most of its requests, one token each, and takes in chunks of the others.
        {"name": "prefill_mixed", "kind": "prefill", "B": 48, "H": 4, "G": 4, "D": 128, "cached": 4096, "low": 0.1,
         "added": 256, "ones": 0.85, "page": 32, "dtype": "bf16", "layout": "nhd"},
        # The paper's width 80 in 32 bits, odd numbers.
        {"name": "prefill_f32", "kind": "prefill", "B": 5, "H": 8, "G": 1, "D": 80, "cached": 777, "low": 0.02,
         "added": 301, "ones": 0.0, "page": 16, "dtype": "f32", "layout": "hnd"},
        # The rows of a decode step, 64 requests, 8 heads of width 80 in one projection's output.
        {"name": "norm_step", "kind": "norm", "B": 1, "T": 64, "Hq": 8, "H": 8, "D": 80, "rope": 80, "order": "half",
         "factor": 1.0, "dtype": "bf16", "weights": "f32"},
        # The rows of a long context's prompt: key heads shared, part of the head turned, pairs side by side, scaled.
        {"name": "norm_prompt", "kind": "norm", "B": 1, "T": 16384, "Hq": 16, "H": 4, "D": 128, "rope": 64,
         "order": "interleaved", "factor": 8.0, "dtype": "bf16", "weights": "bf16"},
        # The backward pass of a training step of the 100M-scale layer.
        {"name": "norm_grad", "kind": "normgrad", "B": 8, "T": 2048, "Hq": 12, "H": 12, "D": 64, "rope": 64,
         "order": "half", "factor": 1.0, "dtype": "bf16", "weights": "f32"},
        # One user's next token and its alternatives, a vocabulary of 32000 in 32 bits.
        {"name": "score_one", "kind": "score", "N": 1, "V": 32000, "K": 5, "dtype": "f32", "slope": 1.2,
         "order": "mixed"},
        # The tokens of a prompt with the most alternatives that are usual, rows not on 16-byte boundaries.
        {"name": "score_prompt", "kind": "score", "N": 1000, "V": 50257, "K": 20, "dtype": "bf16", "slope": 1.1,
         "order": "ranked"},
        # A training step's rows: 16384 tokens of a small vocabulary in 32 bits.
        {"name": "train_small", "kind": "train", "N": 16384, "V": 5003, "K": 0, "dtype": "f32", "slope": 1.1,
         "order": "mixed"},
        # The same with a large vocabulary in bf16.
        {"name": "train_large", "kind": "train", "N": 4096, "V": 131072, "K": 0, "dtype": "bf16", "slope": 1.2,
         "order": "mixed"},
    ]


# ---------------------------------------------------------------------------
# Drawn cases: the same kinds over their ranges
# ---------------------------------------------------------------------------
def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(max(hi, lo))))


def _int(rng, lo, hi):
    return max(lo, min(hi, int(round(_log(rng, lo, hi)))))


def draw(rng):
    kind = rng.choice(["prefill", "prefill", "prefill", "norm", "normgrad", "score", "score", "train"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if kind == "prefill":
        H, G = rng.choice([1, 2, 4, 8, 12, 16]), rng.choice([1, 1, 1, 2, 3, 4, 8])
        most = 1 << (29 if dtype == "bf16" else 27)
        while True:  # the work of a padded batch stays under the largest listed one's
            B, cached, added = _int(rng, 1, 64), _int(rng, 1, 32768) - 1, _int(rng, 1, 4096)
            if B * H * G * added * (cached + added) <= most:
                break
        return {"kind": kind, "B": B, "H": H, "G": G, "D": rng.choice([32, 48, 64, 64, 80, 96, 128]), "cached": cached,
                "low": rng.uniform(0.0, 1.0), "added": added, "ones": rng.choice([0.0, 0.0, 0.5, 0.9]),
                "page": rng.choice([1, 8, 16, 16, 32, 64, 128]), "dtype": dtype, "layout": rng.choice(["hnd", "nhd"])}
    if kind in ("norm", "normgrad"):
        D, H = rng.choice([32, 48, 60, 64, 64, 80, 96, 128]), rng.choice([1, 2, 4, 8, 12])
        Hq = H * rng.choice([1, 1, 2, 4])
        B = rng.choice([1, 1, 2, 8])
        T = _int(rng, 1, (1 << 25) // (B * (Hq + H) * D))
        return {"kind": kind, "B": B, "T": T, "Hq": Hq, "H": H, "D": D, "rope": rng.choice([D, D, D // 4 * 2, 0]),
                "order": rng.choice(["half", "interleaved"]), "factor": rng.choice([1.0, 1.0, 4.0, 8.0]), "dtype": dtype,
                "weights": rng.choice(["f32", "bf16"]) if dtype == "bf16" else "f32"}
    V = _int(rng, 300, 131072)
    N = _int(rng, 1, min(16384, (1 << (26 if kind == "score" else 28)) // V))
    return {"kind": kind, "N": N, "V": V, "K": rng.choice([0, 1, 5, 8, 20, 32]) if kind == "score" else 0, "dtype": dtype,
            "slope": rng.uniform(1.0, 1.6), "order": rng.choice(["mixed", "ranked"])}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _spread(n, lo, hi):
    """n whole numbers spread evenly from lo to hi."""
    return [int(hi)] if n == 1 else [int(round(lo + i * (hi - lo) / (n - 1))) for i in range(n)]


def _requests(c):
    """(cached, added) of each request of a prefill case."""
    B = c["B"]
    cached = _spread(B, math.floor(c["low"] * c["cached"]), c["cached"])
    alone = int(c["ones"] * B)  # requests of one new token
    added = [1] * alone + _spread(B - alone, (1 + c["added"]) // 2, c["added"])
    at = sorted(range(B), key=lambda b: (b * 7919) % 65537)  # short and long histories for either
    return [(cached[b], added[i]) for b, i in zip(range(B), at)]


def _table(lens, page, g, dev):
    """Block tables of requests that hold lens[b] tokens: pages in a random order, -1 past the last; and the pool's
    pages, as many as so many tokens of so many requests can take."""
    used = (lens.long() + page - 1) // page
    W, pool = int(used.max()), (int(lens.sum()) + lens.numel() * (page - 1)) // page + 3
    ids = torch.randperm(pool, device=dev, generator=g)
    col = torch.arange(W, device=dev)[None]
    at = (used.cumsum(0) - used)[:, None] + col
    return torch.where(col < used[:, None], ids[at.clamp(max=pool - 1)], -1).to(torch.int32), pool


def prepare(c, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    s = {"case": c}
    t = DTYPES[c["dtype"]]
    randn = lambda *shape: torch.randn(*shape, device=dev, generator=g, dtype=torch.float32)
    if c["kind"] == "prefill":
        pairs = torch.tensor(_requests(c), device=dev)[torch.randperm(c["B"], device=dev, generator=g)]
        added, lens = pairs[:, 1], pairs.sum(1)
        page, D, H = c["page"], c["D"], c["H"]
        s["most"] = int(added.max())  # new tokens of one request: what the host's own count says
        s["lengths"] = lens.to(torch.int32)
        s["row_start"] = torch.cat([added.new_zeros(1), added.cumsum(0)]).to(torch.int32)
        s["table"], pages = _table(lens, page, g, dev)
        used = torch.zeros(pages, page, dtype=torch.bool, device=dev)
        at = torch.arange(s["table"].shape[1] * page, device=dev)
        slot = s["table"].long().repeat_interleave(page, 1) * page + at % page
        used.view(-1)[slot[at[None] < lens[:, None]]] = True
        for name in ("k_cache", "v_cache"):
            x = randn((pages, page, H, D) if c["layout"] == "nhd" else (pages, H, page, D)).to(t)
            x = x.transpose(1, 2) if c["layout"] == "nhd" else x
            s[name] = x.masked_fill_(~used[:, None, :, None], math.nan)  # what no request holds is whatever was there
        s["q"] = randn(int(added.sum()), H * c["G"], D).to(t)
        s["lam"] = torch.full((1,), 0.5, device=dev)  # the paper's initial value
        return s
    if c["kind"] in ("norm", "normgrad"):
        B, T, Hq, H, D = c["B"], c["T"], c["Hq"], c["H"], c["D"]

        def heads():  # queries and keys as they stand in one projection's output, values behind them
            x = (randn(B, T, Hq + 2 * H, D) * (0.5 + 2.0 * torch.rand(B, T, Hq + 2 * H, 1, device=dev, generator=g))).to(t)
            return x[:, :, :Hq].transpose(1, 2), x[:, :, Hq:Hq + H].transpose(1, 2)

        s["q"], s["k"] = heads()
        s["wq"], s["wk"] = ((1.0 + 0.2 * randn(D)).to(DTYPES[c["weights"]]) for _ in range(2))
        if c["kind"] == "norm":  # the tokens of several requests, each from a place of its own
            first = torch.randint(0, 30000, (B, 1), device=dev, generator=g)
            s["positions"] = (first + torch.arange(T, device=dev)[None] * 7 % 16384).to(torch.int32)
        else:  # whole sequences, all from 0
            s["positions"] = torch.arange(T, device=dev, dtype=torch.int32).expand(B, T)
            s["dq"], s["dk"] = heads()
        s["rope"] = {"rope_dim": c["rope"], "rope_base": ROPE_BASE, "layout": c["order"], "factor": c["factor"],
                     "original_length": 2048 if c["factor"] > 1.0 else 0,
                     "amplitude": 1.0 + 0.1 * math.log(c["factor"])}
        return s
    N, V = c["N"], c["V"]
    rank = torch.rand(N, V, device=dev, generator=g).mul_(V) if c["order"] == "mixed" else \
        torch.arange(V, device=dev, dtype=torch.float32).expand(N, V)
    x = torch.log1p(rank).mul_(-c["slope"])
    x += randn(N, V).mul_(0.3)
    s["logits"] = x.to(t)
    # the tokens that were said: likely ones mostly, and a few places without one (a prompt's end, padding)
    best = torch.argmax(s["logits"], 1)
    said = torch.where(torch.rand(N, device=dev, generator=g) < 0.6, best,
                       torch.randint(0, V, (N,), device=dev, generator=g))
    s["tokens"] = torch.where(torch.rand(N, device=dev, generator=g) < (0.05 if N > 1 else 0.0), -1, said)
    if c["kind"] == "train":  # the losses' own gradients: an advantage for each token, a bonus for entropy
        s["dlogprob"] = randn(N) / N
        s["dentropy"] = torch.full((N,), -0.01 / N, device=dev)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"prefill": _prefill, "norm": _norm, "normgrad": _norm_grad, "score": _score, "train": _train}[kind](s)
    from paper_2608_20172_amd import binding as R
    if kind == "prefill":
        return R.relation_paged_prefill(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["row_start"],
                                        s["lam"])
    if kind == "norm":
        return R.relation_qk_norm_fwd(s["q"], s["k"], s["wq"], s["wk"], s["positions"], eps=EPS, **s["rope"])
    if kind == "normgrad":
        return R.relation_qk_norm_bwd(s["q"], s["k"], s["wq"], s["wk"], s["dq"], s["dk"], s["positions"], eps=EPS,
                                      **s["rope"])
    f = R.relation_token_logprobs_fwd(s["logits"], s["tokens"], top=s["case"]["K"], want_rank=kind == "score")
    if kind == "score":
        return {n: f[n] for n in ("logprob", "entropy", "rank", "top_tokens", "top_logprobs")}
    d = R.relation_token_logprobs_bwd(s["logits"], s["tokens"], f["stats"], s["dlogprob"], s["dentropy"])
    return {"logprob": f["logprob"], "entropy": f["entropy"], "dlogits": d}


def _gathered(x, table, n):
    """[B, H, W page, D] of the pages of each request, zero past its length, in 32 bits."""
    B, W = table.shape
    y = x[table.clamp(min=0).long()].permute(0, 2, 1, 3, 4).reshape(B, x.shape[1], W * x.shape[2], x.shape[3]).float()
    return y.masked_fill_(torch.arange(y.shape[2], device=y.device)[None, None, :, None] >= n[:, None, None, None], 0.0)


def _prefill(s):
    c = s["case"]
    B, H, G, D, most = c["B"], c["H"], c["G"], c["D"], s["most"]
    n, start = s["lengths"].long(), s["row_start"].long()
    K, V = _gathered(s["k_cache"], s["table"], n), _gathered(s["v_cache"], s["table"], n)
    N = s["q"].shape[0]
    r = torch.arange(most, device=n.device)
    mine = r[None] < (start[1:] - start[:-1])[:, None]  # [B, most]
    row = (start[:-1, None] + r[None]).clamp(max=N - 1)
    q = (s["q"].float() / math.sqrt(D))[row].view(B, most, H, G, D).permute(0, 2, 4, 1, 3).reshape(B, H, D, most * G)
    U = K @ q.contiguous()  # [B, H, T, most G]
    at = (n[:, None] - (start[1:] - start[:-1])[:, None] + r[None]).clamp(max=K.shape[2] - 1)  # positions from 0
    at = at[:, :, None].expand(B, most, G).reshape(B, 1, 1, most * G)
    S = torch.sigmoid(torch.gather(U, 2, at.expand(B, H, 1, most * G)) / TAU)
    later = torch.arange(K.shape[2], device=n.device)[None, None, :, None] >= at
    E = (U * torch.sigmoid(U)).masked_fill_(later, -math.inf)
    del U
    m = E.amax(2, keepdim=True).clamp(min=-3.0e38)
    P = torch.exp(E - m)
    del E
    l = P.sum(2, keepdim=True)
    ln = torch.log((at + 1).float())
    A = torch.log(l) + m - s["lam"] * ln
    z = P.transpose(2, 3).contiguous() @ V  # [B, H, most G, D]
    vi = torch.gather(V, 2, at.transpose(2, 3).expand(B, H, most * G, D))
    col = lambda x: x.transpose(2, 3)
    y = torch.sigmoid(col(S - A)) * vi + torch.sigmoid(col(A - S)) * (z / col(l).clamp(min=1.0e-30))
    top = torch.maximum(S, A)
    M = top + torch.log(torch.exp(S - top) + torch.exp(A - top)) + s["lam"] * ln
    y = y.view(B, H, most, G, D).permute(0, 2, 1, 3, 4).reshape(B, most, H * G, D)[mine]
    M = M.view(B, H, most, G).permute(0, 2, 1, 3).reshape(B, most, H * G)[mine]
    return {"o": y.to(s["q"].dtype), "row_stat": M}


def _turns(s):
    """cos and sin times the amplitude, [B, 1, T, rope / 2]; angles in 64 bits: a position times a frequency leaves
    nothing of 32 bits' fraction in a long context."""
    p = s["rope"]
    w = p["rope_base"] ** (-2.0 * torch.arange(p["rope_dim"] // 2, dtype=torch.float64, device=s["q"].device) /
                           max(p["rope_dim"], 1))
    # frequencies that turn 32 times or more within the original length stay, those under once are divided by the factor
    keep = ((p["original_length"] * w / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    ang = s["positions"].double()[:, None, :, None] * (w * (keep + (1.0 - keep) / p["factor"]))
    return (torch.cos(ang) * p["amplitude"]).float(), (torch.sin(ang) * p["amplitude"]).float()


def _halves(x, p):
    d = p["rope_dim"]
    return (x[..., 0:d:2], x[..., 1:d:2]) if p["layout"] == "interleaved" else (x[..., :d // 2], x[..., d // 2:d])


def _joined(a, b, rest, p):
    y = torch.stack([a, b], -1).flatten(-2) if p["layout"] == "interleaved" else torch.cat([a, b], -1)
    return torch.cat([y, rest], -1)


def _norm(s):
    p, (cs, sn) = s["rope"], _turns(s)
    out = {}
    for name, w in (("q", "wq"), ("k", "wk")):
        x = s[name].float()
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s[w].float()
        a, b = _halves(x, p)
        out[name] = _joined(a * cs - b * sn, a * sn + b * cs, x[..., p["rope_dim"]:], p).to(s[name].dtype)
    return out


def _norm_grad(s):
    p, (cs, sn) = s["rope"], _turns(s)
    out = {}
    for name, w in (("q", "wq"), ("k", "wk")):
        x, g = s[name].float(), s["d" + name].float()
        a, b = _halves(g, p)
        g = _joined(a * cs + b * sn, b * cs - a * sn, g[..., p["rope_dim"]:], p)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        xr = x * r
        out["d" + w] = (g * xr).sum((0, 1, 2))
        g = g * s[w].float()
        out["d" + name] = (r * (g - xr * (g * xr).mean(-1, keepdim=True))).to(s[name].dtype)
    return out


def _stats(s):
    x = s["logits"].float()
    d = x - x.amax(1, keepdim=True)
    w = torch.exp(d)
    Z = w.sum(1, keepdim=True)
    lnZ = torch.log(Z)
    H = (lnZ - (w * d).sum(1, keepdim=True) / Z)[:, 0]
    t = s["tokens"].clamp(min=0)[:, None]
    return d, lnZ, H, torch.where(s["tokens"] < 0, 0.0, (d.gather(1, t) - lnZ)[:, 0])


def _score(s):
    d, lnZ, H, lp = _stats(s)
    x, K = s["logits"].float(), s["case"]["K"]
    t = s["tokens"].clamp(min=0)[:, None]
    xt = x.gather(1, t)
    before = (x > xt) | ((x == xt) & (torch.arange(x.shape[1], device=x.device)[None] < t))
    rank = torch.where(s["tokens"] < 0, -1, before.sum(1))
    at = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :K]  # ties: lower index first
    return {"logprob": lp, "entropy": H, "rank": rank.to(torch.int32), "top_tokens": at,
            "top_logprobs": d.gather(1, at) - lnZ}


def _train(s):
    d, lnZ, H, lp = _stats(s)
    logp = d - lnZ
    p = torch.exp(logp)
    grad = -p * (torch.where(s["tokens"] < 0, 0.0, s["dlogprob"])[:, None] + s["dentropy"][:, None] * (logp + H[:, None]))
    grad.scatter_add_(1, s["tokens"].clamp(min=0)[:, None], torch.where(s["tokens"] < 0, 0.0, s["dlogprob"])[:, None])
    return {"logprob": lp, "entropy": H, "dlogits": grad.to(s["logits"].dtype)}


# ---------------------------------------------------------------------------
# The work that a pass cannot do without
# ---------------------------------------------------------------------------
def work(c):
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "prefill":
        reqs = _requests(c)
        keys, new = sum(a + n for a, n in reqs), sum(n for _, n in reqs)
        pairs = sum(n * a + n * (n + 1) / 2.0 for a, n in reqs)
        Hq = c["H"] * c["G"]
        # K and V rows of every entry and the page ids; q in, o and row_stat out
        return {"bytes": 2 * c["H"] * keys * c["D"] * es + 4 * keys / c["page"] + 2 * new * Hq * c["D"] * es +
                4 * new * Hq + 8 * c["B"], "flops": 4.0 * Hq * pairs * c["D"]}
    if c["kind"] in ("norm", "normgrad"):
        n = c["B"] * c["T"] * (c["Hq"] + c["H"]) * c["D"]
        tensors, ops = (2, 6.0) if c["kind"] == "norm" else (3, 12.0)
        return {"bytes": tensors * n * es + 4 * c["T"], "flops": ops * n}
    n = c["N"] * c["V"]
    if c["kind"] == "score":
        return {"bytes": n * es + c["N"] * (20 + 12 * c["K"]), "flops": 4.0 * n}
    return {"bytes": 2 * n * es + 24 * c["N"], "flops": 9.0 * n}


# ---------------------------------------------------------------------------
# The same outputs in 64 bits
# ---------------------------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    f = torch.float64
    if c["kind"] == "prefill":
        H, G, page, D = c["H"], c["G"], c["page"], c["D"]
        dev = s["q"].device
        o = torch.empty(s["q"].shape, dtype=f, device=dev)
        M = torch.empty(s["q"].shape[:2], dtype=f, device=dev)
        lam, start = float(s["lam"][0]), s["row_start"].tolist()
        for b, n in enumerate(s["lengths"].tolist()):
            ids = s["table"][b, : (n + page - 1) // page].long()
            rows = slice(start[b], start[b + 1])
            i = torch.arange(n - (start[b + 1] - start[b]), n, device=dev)[:, None]  # positions from 0
            j = torch.arange(n, device=dev)[None]
            for h in range(H):
                k, v = (s[x][ids, h].reshape(-1, D)[:n].to(f) for x in ("k_cache", "v_cache"))
                for r in range(h * G, (h + 1) * G):
                    U = s["q"][rows, r].to(f) @ k.T.contiguous() / math.sqrt(D)
                    R = U / (1.0 + torch.exp(-U)) - lam * torch.log((i + 1).to(f))
                    R = torch.where(j == i, 1.0 / (1.0 + torch.exp(-U / TAU)), R).masked_fill_(j > i, -math.inf)
                    lse = torch.logsumexp(R, 1)
                    o[rows, r] = torch.exp(R - lse[:, None]) @ v
                    M[rows, r] = lse + lam * torch.log((i[:, 0] + 1).to(f))
        return {"o": o, "row_stat": M}
    if c["kind"] in ("norm", "normgrad"):
        p, D = s["rope"], c["D"]
        d = p["rope_dim"]
        w = torch.exp(-math.log(p["rope_base"]) * torch.arange(0, d, 2, device=s["q"].device, dtype=f) / max(d, 1))
        if p["factor"] != 1.0:
            often = p["original_length"] * w / (2 * math.pi)  # rotations within the original length
            share = torch.minimum(torch.maximum((often - 1) / (32 - 1), torch.zeros_like(w)), torch.ones_like(w))
            w = share * w + (1 - share) * w / p["factor"]
        turn = p["amplitude"] * torch.exp(1j * s["positions"].to(f)[:, None, :, None] * w)

        def turned(x, by):
            a, b = (x[..., 0:d:2], x[..., 1:d:2]) if p["layout"] == "interleaved" else (x[..., :d // 2], x[..., d // 2:d])
            z = torch.complex(a.contiguous(), b.contiguous()) * by
            y = x.clone()
            if p["layout"] == "interleaved":
                y[..., 0:d:2], y[..., 1:d:2] = z.real, z.imag
            else:
                y[..., :d // 2], y[..., d // 2:d] = z.real, z.imag
            return y

        out = {}
        for name, wn in (("q", "wq"), ("k", "wk")):
            x, wt = s[name].to(f), s[wn].to(f)
            rms = torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS)
            if c["kind"] == "norm":
                out[name] = turned(x / rms * wt, turn)
                continue
            g = turned(s["d" + name].to(f), turn.conj())
            out["d" + wn] = torch.einsum("bhtd,bhtd->d", g, x / rms)
            g = g * wt
            out["d" + name] = g / rms - x * (g * x).sum(-1, keepdim=True) / (D * rms ** 3)
        return out
    N, V, K = c["N"], c["V"], c["K"]
    res = {"logprob": torch.empty(N, dtype=f, device=s["logits"].device)}
    res["entropy"] = torch.empty_like(res["logprob"])
    if c["kind"] == "score":
        res |= {"rank": None, "top_tokens": None, "top_logprobs": res["logprob"].new_empty(N, K)}
    else:
        res["dlogits"] = torch.empty(N, V, dtype=f, device=s["logits"].device)
    for a in range(0, N, 512):  # rows at a time
        b = slice(a, min(a + 512, N))
        logp = torch.log_softmax(s["logits"][b].to(f), 1)
        p = torch.exp(logp)
        said = s["tokens"][b] >= 0
        one = torch.zeros_like(p).scatter_(1, s["tokens"][b].clamp(min=0)[:, None], 1.0) * said[:, None]
        res["logprob"][b] = (one * logp).sum(1)
        res["entropy"][b] = -(p * logp).sum(1)
        if c["kind"] == "score":
            res["top_logprobs"][b] = torch.topk(logp, K, 1)[0]
        else:
            bits = -(p * logp).sum(1, keepdim=True)
            res["dlogits"][b] = s["dlogprob"][b].to(f)[:, None] * (one - p * said[:, None]) - \
                s["dentropy"][b].to(f)[:, None] * p * (logp + bits)
    return res
