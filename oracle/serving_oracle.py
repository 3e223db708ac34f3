"""fp64 CPU oracle of the serving operators: page maps, rows into a paged cache,
the decode step over pages, and sampling.

TEST INFRASTRUCTURE. Only the tests may import this module. The product path
never calls it, and it shares no code with that path. Everything is written
request by request and token by token from the definitions in
``include/relation.h``: page maps and samples are whole numbers and have to be
met exactly, the rest within rounding.
"""
from __future__ import annotations

import math

import numpy as np

from .decode_oracle import decode_step
from .layer_oracle import givens
from .relation_oracle import TAU_S

__all__ = ["page_map", "turned", "append", "paged_decode", "sample"]


def page_map(cached, added, table, free_pages, page_size: int, max_tokens: int) -> dict:
    """One request after another: who is served, with which pages and slots."""
    table = np.array(table, np.int64)
    B, W = table.shape
    lengths, row_start = np.zeros(B, np.int64), np.zeros(B + 1, np.int64)
    slots, positions = np.full(max_tokens, -1, np.int64), np.full(max_tokens, -1, np.int64)
    at = 0        # where the request's tokens start
    wanted = 0    # pages that it and those before it need
    taken = mapped = refused = 0
    for b in range(B):
        c, n = int(cached[b]), int(added[b])
        tokens = max(n, 0)
        row_start[b + 1] = min(at + tokens, max_tokens)
        have, want = -(-max(c, 0) // page_size), -(-(c + n) // page_size)
        ok = c >= 0 and n >= 0 and want <= W
        need = want - have if ok else 0
        wanted += need
        ok = ok and (tokens == 0 or at + tokens <= max_tokens) and (need == 0 or wanted <= len(free_pages))
        if ok:
            for j in range(need):
                table[b, have + j] = free_pages[wanted - need + j]
            for t in range(n):
                pos = c + t
                slots[at + t] = table[b, pos // page_size] * page_size + pos % page_size
                positions[at + t] = pos
            lengths[b] = c + n
            taken += need
            mapped += n
        else:
            refused += 1
        at += tokens
    return {"table": table, "lengths": lengths, "row_start": row_start, "slots": slots, "positions": positions,
            "counts": np.array([taken, mapped, refused])}


def turned(x, position: int, base: float):
    """x [..., D] with channel d turned with channel d + D/2 by the angle position base^(-2d/D), as a complex phase."""
    x = np.asarray(x, np.float64)
    h = x.shape[-1] // 2
    z = (x[..., :h] + 1j * x[..., h:]) * np.exp(1j * position * base ** (-2.0 * np.arange(h) / x.shape[-1]))
    return np.concatenate([z.real, z.imag], -1)


def append(k, v, k_cache, v_cache, slots, positions, *, q=None, theta=None, pairing=None, rope_base=1.0e4):
    """Caches [pages, H, page, Dc] with the rows of k, v [N, H, D] in them, and the rotated, padded q (or None)."""
    k_cache, v_cache = np.array(k_cache, np.float64), np.array(v_cache, np.float64)
    P, H, page, Dc = k_cache.shape
    N, _, D = k.shape
    pad = lambda x: np.concatenate([x, np.zeros(x.shape[:-1] + (Dc - D,))], -1)
    row = lambda x, n: turned(x[n], int(positions[n]), rope_base) if rope_base else np.asarray(x[n], np.float64)
    q_out = None if q is None else np.zeros(q.shape[:2] + (Dc,))
    mixed = np.asarray(v, np.float64)
    if pairing is not None:
        mixed = givens(mixed.transpose(1, 0, 2)[None], np.asarray(theta, np.float64), pairing)[0].transpose(1, 0, 2)
    for n in range(N):
        if slots[n] < 0 or positions[n] < 0 or slots[n] >= P * page:
            continue
        p, r = divmod(int(slots[n]), page)
        k_cache[p, :, r] = pad(row(k, n))
        v_cache[p, :, r] = pad(mixed[n])
        if q is not None:
            q_out[n] = pad(row(q, n))
    return k_cache, v_cache, q_out


def paged_decode(q, k_cache, v_cache, table, lengths, lam, *, tau_s: float = TAU_S, scale=None, max_length=None):
    """y [B, Hq, D] and M [B, Hq]; NaN for a request with a bad length or page."""
    P, H, page, D = k_cache.shape
    B, Hq, _ = q.shape
    W = np.shape(table)[1]
    cap = min(W * page, max_length or W * page)
    Y, M = np.full((B, Hq, D), np.nan), np.full((B, Hq), np.nan)
    for b in range(B):
        n = int(lengths[b])
        ids = [int(x) for x in table[b][: -(-n // page)]] if 1 <= n <= cap else []
        if not ids or min(ids) < 0 or max(ids) >= P:
            continue
        for h in range(Hq):
            k = k_cache[ids, h * H // Hq].reshape(-1, D)[:n]
            v = v_cache[ids, h * H // Hq].reshape(-1, D)[:n]
            Y[b, h], M[b, h] = decode_step(q[b, h], k, v, n, lam, tau_s=tau_s, scale=scale)
    return Y, M


def sample(x, noise, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row of logits: dict(token, logprob, kept (the kept tokens in order), lead: the relative distance of the
    race's second from its winner)."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if not (temperature >= 0) or math.isnan(top_p) or math.isnan(min_p) or top == -np.inf:
        return {"token": -1, "logprob": math.nan, "kept": [], "lead": math.inf}
    T, k = (1.0, 1) if temperature == 0 else (float(temperature), int(top_k) if top_k > 0 else len(x))
    with np.errstate(invalid="ignore", over="ignore"):  # -inf, and what is finite beside +inf, weighs nothing at any T
        d = np.where(x == top, 0.0, np.where(x - top == -np.inf, -np.inf, (x - top) / T))
    w = np.exp(d)
    Z = math.fsum(w)
    order = np.lexsort((np.arange(len(x)), -x))  # falling x, then the index
    before = np.concatenate([[0.0], np.cumsum(w[order])[:-1]])
    keep = (np.arange(len(x)) < k) & ((top_p >= 1) | (before < top_p * Z)) & (w[order] >= min_p)
    keep[0] = True
    kept = order[keep]
    score = w[kept] / np.maximum(np.asarray(noise, np.float64)[kept], 2.0 ** -126)
    best = score.max()
    token = int(kept[score == best].min())
    others = score[kept != token]
    lead = (best - others.max()) / best if others.size else math.inf
    return {"token": token, "logprob": d[token] - math.log(Z), "kept": kept.tolist(), "lead": lead}
