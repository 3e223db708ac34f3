#!/usr/bin/env python3
"""Generate tokens for several requests from one paged cache.

A small Relation decoder with random weights takes in prompts of different
lengths, whole or in chunks, and then decodes them together, one token each a step:

  relation_page_map        pages and slots of the step's tokens, from lengths on the GPU
  relation_qk_norm_fwd     RMS norm of the heads of q and k and RoPE (--norm)
  relation_paged_append    RoPE on q and k without --norm, Givens mixing of v, rows into the pages
  relation_paged_prefill   Full Relation of the prompts' rows over the pages
  relation_paged_decode    the same of one new row of each request
  relation_token_logprobs_fwd  log-probability and rank of the prompts' own tokens
  relation_sample          the next tokens from the logits

Every layer has its own pools; the block tables are shared. The host keeps count
of what it asks for and reads nothing back but the finished tokens.

  python examples/serve_paged.py [--steps N] [--chunk N] [--norm] [--check]

--check replays the finished sequences through relation_layer_fwd and compares
the last hidden rows with those of the decode steps.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_20172_amd import binding as R  # noqa: E402


class Decoder:
    """Layers of norm, q/k/v projections, Relation and an output projection, with a residual; random weights. With
    head_norm, q and k have an RMS norm of every head, with weights, before the rotation."""

    def __init__(self, vocab=5000, layers=2, heads=8, width=64, seed=0, dev="cuda", head_norm=False):
        g = torch.Generator(device=dev).manual_seed(seed)
        dim = heads * width
        mat = lambda n, m: (torch.randn(n, m, device=dev, generator=g) / n ** 0.5).to(torch.bfloat16)
        self.H, self.D, self.dim, self.layers = heads, width, dim, layers
        self.emb, self.head = mat(vocab, dim) * vocab ** 0.5, mat(dim, vocab) * 4
        self.wqkv = [mat(dim, 3 * dim) for _ in range(layers)]
        self.wo = [mat(dim, dim) for _ in range(layers)]
        self.lam = [torch.full((1,), 0.5, device=dev) for _ in range(layers)]
        self.theta = [(torch.rand(heads // 2, device=dev, generator=g) * 2 - 1) for _ in range(layers)]
        self.pairing = ["A" if n % 2 == 0 else "B" for n in range(layers)]
        weight = lambda: 1 + 0.3 * torch.randn(width, device=dev, generator=g)
        self.head_norms = [(weight(), weight()) for _ in range(layers)] if head_norm else None

    def qkv(self, n, x):
        """q, k, v [N, H, D] of x [N, dim]."""
        y = x.float()
        y = (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)
        return (y @ self.wqkv[n]).view(-1, 3, self.H, self.D).unbind(1)

    def whole(self, tokens):
        """Hidden rows [T, dim] of one sequence, every row by relation_layer_fwd."""
        x = self.emb[tokens]
        for n in range(self.layers):
            q, k, v = (t.transpose(0, 1)[None] for t in self.qkv(n, x))
            if self.head_norms:
                f = R.relation_qk_norm_fwd(q, k, *self.head_norms[n], rope_dim=0)
                q, k = f["q"], f["k"]
            o = R.relation_layer_fwd(q, k, v, self.lam[n], self.theta[n], pairing=self.pairing[n])["o"]
            x = x + o[0].transpose(0, 1).reshape(-1, self.dim) @ self.wo[n]
        return x


class Pool:
    """The caches of all layers, the block tables of B requests, and the free pages."""

    def __init__(self, model, requests, pages, page_size, max_length, dev="cuda"):
        width = -(-model.D // 8) * 8  # the caches' rows are multiples of 16 bytes; narrower heads are padded
        shape = (model.layers, pages, 2, model.H, page_size, width)
        self.kv = torch.zeros(shape, dtype=torch.bfloat16, device=dev)
        self.table = torch.full((requests, -(-max_length // page_size)), -1, dtype=torch.int32, device=dev)
        self.free = torch.randperm(pages, device=dev).to(torch.int32)
        self.lengths = torch.zeros(requests, dtype=torch.int32, device=dev)
        self.page_size = page_size
        self.count, self.taken = [0] * requests, 0  # the host's own: tokens of each request, pages given out

    def caches(self, layer):
        return self.kv[layer, :, 0], self.kv[layer, :, 1]

    def step(self, added):
        """Pages and slots for added[b] more tokens of each request. Raises, and changes nothing, where they do not fit:
        the map gives a request that it cannot serve length 0, and a loop that fed that back would start it over."""
        now = [c + a for c, a in zip(self.count, added)]
        need = sum(-(-n // self.page_size) + -c // self.page_size for n, c in zip(now, self.count))
        if self.taken + need > len(self.free) or max(now) > self.table.shape[1] * self.page_size:
            raise RuntimeError(f"{need} pages needed, {len(self.free) - self.taken} free; up to {max(now)} tokens of a "
                               f"request, a table row holds {self.table.shape[1] * self.page_size}")
        m = R.relation_page_map(self.lengths, torch.tensor(added, dtype=torch.int32, device=self.table.device), self.table,
                                self.free[self.taken:], self.page_size, sum(added))
        self.lengths, self.count, self.taken = m["lengths"], now, self.taken + need
        return m


def new_rows(model, pool, m, x, one_each, longest):
    """Hidden rows [N, dim] of a step's tokens (x: their embeddings), whose keys and values go into the pages; one_each:
    the step has one token of every request."""
    for n in range(model.layers):
        q, k, v = model.qkv(n, x)
        base = R.ROPE_BASE
        if model.head_norms:
            f = R.relation_qk_norm_fwd(q, k, *model.head_norms[n], m["positions"])
            q, k, base = f["q"], f["k"], None
        caches = pool.caches(n)
        q = R.relation_paged_append(k, v, *caches, m["slots"], m["positions"], q=q, theta=model.theta[n],
                                    pairing=model.pairing[n], rope_base=base)
        over = (m["lengths"],) if one_each else (m["lengths"], m["row_start"])
        f = (R.relation_paged_decode if one_each else R.relation_paged_prefill)(
            q, *caches, pool.table, *over, model.lam[n], max_length=longest, head_dim=model.D)
        x = x + f["o"][:, :, :model.D].reshape(-1, model.dim) @ model.wo[n]
    return x


def take_in(model, pool, prompts, longest, chunk=None):
    """The prompts, up to `chunk` tokens of each a step: the hidden rows [T, dim] of each."""
    if chunk is not None and chunk < 1:
        raise ValueError("a chunk has at least one token")
    rows, at = [[] for _ in prompts], 0
    while at < max(len(p) for p in prompts):
        part = [p[at:at + (chunk or longest)] for p in prompts]
        added = [len(p) for p in part]
        x = new_rows(model, pool, pool.step(added), model.emb[torch.cat(part)], False, longest)
        for r, y in zip(rows, x.split(added)):
            r.append(y)
        at += max(added)
    return [torch.cat(r) for r in rows]


def score(model, prompts, rows):
    """Log-probability and rank [T - 1] of the tokens 1 .. T-1 of each prompt, from its hidden rows."""
    tokens = torch.cat([torch.cat([p[1:], p.new_full((1,), -1)]) for p in prompts])  # -1: none given after the last
    f = R.relation_token_logprobs_fwd(torch.cat(rows) @ model.head, tokens, want_rank=True)
    at = [len(p) for p in prompts]
    return [(a[:-1], b[:-1]) for a, b in zip(f["logprob"].split(at), f["rank"].split(at))]


def sample(model, x, g, filters):
    logits = x @ model.head
    noise = torch.empty(logits.shape, device=logits.device).exponential_(generator=g)
    return R.relation_sample(logits, noise, **filters)


def generate(model, prompts, steps, *, page_size=16, seed=1, chunk=None, scores=None, **filters):
    """Token ids [B, steps], their logprobs, and the hidden rows [B, dim] of the last step. scores: a list that gets each
    prompt's own log-probabilities and ranks."""
    dev, B = model.emb.device, len(prompts)
    g = torch.Generator(device=dev).manual_seed(seed)
    longest = max(len(p) for p in prompts) + steps
    pool = Pool(model, B, sum(-(-(len(p) + steps) // page_size) for p in prompts), page_size, longest)
    rows = take_in(model, pool, prompts, longest, chunk)
    if scores is not None:
        scores += score(model, prompts, rows)
    x = torch.stack([r[-1] for r in rows])
    out, logprob = [], []
    for step in range(steps):
        s = sample(model, x, g, filters)
        out.append(s["tokens"])
        logprob.append(s["logprob"])
        if step + 1 == steps:
            break
        x = new_rows(model, pool, pool.step([1] * B), model.emb[s["tokens"]], True, longest)
    return torch.stack(out, 1), torch.stack(logprob, 1), x


def check(model, prompts, tokens, x):
    """Relative 2-norm of the last hidden rows against those of the whole sequences."""
    worst = 0.0
    for b, p in enumerate(prompts):
        want = model.whole(torch.cat([p, tokens[b, :-1]]))[-1].float()
        worst = max(worst, float((x[b].float() - want).norm() / want.norm()))
    return worst


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--chunk", type=int, help="take the prompts in by chunks of so many tokens")
    ap.add_argument("--norm", action="store_true", help="RMS norm of the heads of q and k")
    ap.add_argument("--check", action="store_true")
    a = ap.parse_args()
    model = Decoder(head_norm=a.norm)
    g = torch.Generator(device="cuda").manual_seed(3)
    prompts = [torch.randint(0, model.emb.shape[0], (n,), device="cuda", generator=g) for n in (1, 7, 16, 45, 130, 300)]
    scores = []
    tokens, logprob, x = generate(model, prompts, a.steps, chunk=a.chunk, scores=scores, temperature=0.8, top_k=50, top_p=0.9)
    for p, t, l, (own, rank) in zip(prompts, tokens.tolist(), logprob.mean(1).tolist(), scores):
        of_its_own = f", its own {own.mean():.3f}, best rank {int(rank.min())}" if len(p) > 1 else ""
        print(f"prompt of {len(p):4d}: {' '.join(map(str, t[:10]))} ...  mean logprob {l:.3f}{of_its_own}")
    if a.check:
        err = check(model, prompts, tokens, x)
        print(f"last hidden rows against whole sequences: relative 2-norm {err:.2e}")
        if not err < 2e-2:
            raise SystemExit("the paged cache and the whole sequence disagree")


if __name__ == "__main__":
    main()
