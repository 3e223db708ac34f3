"""fp64 CPU oracle of the operators that go token by token: norms and rotation of
query and key heads, and log-probabilities of given tokens, with their gradients.

TEST INFRASTRUCTURE. Only the tests may import this module. The product path
never calls it, and it shares no code with that path. Everything is written from
the definitions in ``include/relation.h``, a row at a time.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["frequencies", "rotation", "norm_rope", "norm_rope_backward", "logprobs", "logprobs_backward"]


def frequencies(rope_dim: int, base: float = 1.0e4, factor: float = 1.0, original_length: int = 0, low: float = 1.0,
                high: float = 32.0):
    """Radians a position of each channel pair."""
    w = []
    for j in range(rope_dim // 2):
        v = base ** (-2.0 * j / rope_dim)
        often = original_length * v / (2.0 * math.pi)
        c = 0.0 if original_length == 0 else min(max((often - low) / (high - low), 0.0), 1.0)
        w.append(v * (c + (1.0 - c) / factor))
    return w


def rotation(D: int, rope_dim: int, position: int, layout: str = "half", amplitude: float = 1.0, **kw):
    """The D x D matrix that turns a row at a position."""
    R = np.eye(D)
    for j, w in enumerate(frequencies(rope_dim, **kw)):
        a, b = (2 * j, 2 * j + 1) if layout == "interleaved" else (j, j + rope_dim // 2)
        c, s = amplitude * math.cos(position * w), amplitude * math.sin(position * w)
        R[a, a], R[a, b], R[b, a], R[b, b] = c, -s, s, c
    return R


def norm_rope(x, weight, positions, *, norm: bool = True, eps: float = 1.0e-6, rope_dim=None, **kw):
    """x [B, H, T, D], positions [B, T]."""
    x = np.asarray(x, np.float64)
    B, H, T, D = x.shape
    w = np.ones(D) if weight is None else np.asarray(weight, np.float64)
    y = np.zeros_like(x)
    for b in range(B):
        for t in range(T):
            if positions[b, t] < 0:
                continue
            R = rotation(D, D if rope_dim is None else rope_dim, int(positions[b, t]), **kw)
            for h in range(H):
                r = x[b, h, t]
                n = r * w / math.sqrt(np.mean(r * r) + eps) if norm else r
                y[b, h, t] = R @ n
    return y


def norm_rope_backward(x, weight, positions, dy, *, norm: bool = True, eps: float = 1.0e-6, rope_dim=None, **kw):
    """(dx, dweight) through the Jacobian of each row: d n_i / d x_j = w_i (delta_ij / s - x_i x_j / (D s^3))."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    B, H, T, D = x.shape
    w = np.ones(D) if weight is None else np.asarray(weight, np.float64)
    dx, dw = np.zeros_like(x), np.zeros(D)
    for b in range(B):
        for t in range(T):
            if positions[b, t] < 0:
                continue
            R = rotation(D, D if rope_dim is None else rope_dim, int(positions[b, t]), **kw)
            for h in range(H):
                r, g = x[b, h, t], R.T @ dy[b, h, t]
                if not norm:
                    dx[b, h, t] = g
                    continue
                s = math.sqrt(np.mean(r * r) + eps)
                J = w[:, None] * (np.eye(D) / s - np.outer(r, r) / (D * s ** 3))
                dx[b, h, t] = J.T @ g
                dw += g * r / s
    return dx, dw


def logprobs(x, token: int, top: int = 0) -> dict:
    """One row of logits: logprob, entropy, rank, the first `top` tokens and their log-probabilities, and all of them."""
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    V, m = len(x), x.max()
    nan = math.nan
    if m == -np.inf:
        return {"logprob": 0.0 if token < 0 else nan, "entropy": nan, "rank": -1, "top_tokens": [-1] * top, "top_logprobs": [nan] * top,
                "logp": np.full(V, nan), "p": np.full(V, nan)}
    with np.errstate(invalid="ignore"):
        d = np.where(x == m, 0.0, x - m)
    p = np.exp(d)
    Z = math.fsum(p)
    logp, p = d - math.log(Z), p / Z
    order = np.lexsort((np.arange(V), -x))  # falling x, then the index
    H = -math.fsum(p[p > 0] * logp[p > 0])
    given = 0 <= token < V
    return {"logprob": logp[token] if given else 0.0 if token < 0 else nan, "entropy": H,
            "rank": int(np.nonzero(order == token)[0][0]) if given else -1, "top_tokens": order[:top].tolist(),
            "top_logprobs": logp[order[:top]].tolist(), "logp": logp, "p": p}


def logprobs_backward(x, token: int, g: float, h: float):
    """d(g logprob + h entropy) / dx through the Jacobian of log-softmax: dlogp_i / dx_j = [i = j] - p_j."""
    r = logprobs(x, token)
    p, logp = r["p"], r["logp"]
    V = len(p)
    if token >= V:
        return np.full(V, math.nan)
    if token < 0 and h == 0:
        return np.zeros(V)  # nothing of the row is asked for
    some = p > 0
    dlogp = np.zeros(V)  # of g logp_t - h sum p logp by logp, with p = exp(logp)
    dlogp[some] = -h * p[some] * (logp[some] + 1.0)
    if token >= 0:
        dlogp[token] += g
    return dlogp - p * math.fsum(dlogp)
