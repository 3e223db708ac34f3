"""Norms of heads, paged chunks and log-probabilities of tokens together, as a serving step and a training step use
them, and the serving example's chunks, norms and scores."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from examples import serve_paged as E
from oracle import relation_oracle as RO
from oracle import serving_oracle as SO
from oracle import token_oracle as TO
from paper_2608_20172_amd import binding as R
from tests.gpu_helpers import log, rel_l2

pytestmark = pytest.mark.gpu

DEV = "cuda"

# Hidden rows of the example, whole sequences and paged steps rounding at other places: relative 2^-8 a rounding, eight
# of them over two layers and two more a layer for the normed heads, at their square root and doubled.
BAR = 2.0 ** -8 * 12 ** 0.5 * 2


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    R.load_library()


def _np(t):
    return t.detach().double().cpu().numpy()


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("D,G,width", [(64, 2, 64), (36, 1, 40)])
def test_serving_step_in_32_bits(D, G, width):
    """Two steps of three requests from projections to log-probabilities, against the oracles in 64 bits.

    Bars: normed rows are at most 2 D^(1/2) long (weights to 1.9), so evidence is at most 4 D^(1/2), 32, and its fp32
    error (2^-20 of the rows' norms, and the products) at most 32 2^-18 = 1.2e-4, of a weight, of a row: 2^1/2 times that
    with the scan's own 2e-5 is under 2e-4. A logit moves by the row's error times its column's length, a log-probability
    by twice the largest such move."""
    rng = np.random.default_rng(3 + D)
    H, page, V, B = 3, 16, 501, 3
    Hq = H * G
    mk = lambda *s, std=1.0: torch.from_numpy(rng.standard_normal(s) * std).float().to(DEV)
    kc, vc = (torch.zeros((20, H, page, width), device=DEV) for _ in range(2))
    okc, ovc = _np(kc), _np(vc)
    wq, wk = (torch.from_numpy(rng.uniform(0.3, 1.9, D)).float().to(DEV) for _ in range(2))
    head = mk(Hq * D, V, std=1.0 / math.sqrt(Hq * D))
    table, free = torch.full((B, 8), -1, dtype=torch.int32, device=DEV), _i32(rng.permutation(20))
    lengths, taken = _i32(np.zeros(B)), 0
    for added in ([33, 1, 70], [5, 40, 1]):
        N = sum(added)
        x = mk(N, Hq + 2 * H, D)
        q, k, v = x.split((Hq, H, H), 1)
        tokens = torch.from_numpy(rng.integers(0, V, N)).to(DEV)
        m = R.relation_page_map(lengths, _i32(added), table, free[taken:], page, N)
        taken += int(m["counts"][0])
        lengths = m["lengths"]
        f = R.relation_qk_norm_fwd(q, k, wq, wk, m["positions"])
        qp = R.relation_paged_append(f["k"], v, kc, vc, m["slots"], m["positions"], q=f["q"], rope_base=None)
        o = R.relation_paged_prefill(qp, kc, vc, table, m["lengths"], m["row_start"], 0.4, head_dim=D)["o"]
        y = o[:, :, :D].reshape(N, Hq * D)
        lp = R.relation_token_logprobs_fwd(y @ head, tokens)["logprob"]
        torch.cuda.synchronize()
        pos = m["positions"].cpu().numpy()
        heads = lambda t, w: TO.norm_rope(_np(t).transpose(1, 0, 2)[None], _np(w), pos[None])[0].transpose(1, 0, 2)
        okc, ovc, oq = SO.append(heads(k, wk), _np(v), okc, ovc, m["slots"].cpu().numpy(), pos, q=heads(q, wq), rope_base=None)
        Y, _ = SO.paged_prefill(oq, okc, ovc, table.cpu().numpy(), lengths.cpu().numpy(), m["row_start"].cpu().numpy(),
                                float(np.float32(0.4)), scale=D ** -0.5)
        Y = np.stack(Y)[:, :, :D].reshape(N, -1)
        W = _np(head)
        want = np.array([TO.logprobs(Y[n] @ W, int(tokens[n]))["logprob"] for n in range(N)])
        err, bar = rel_l2(_np(y), Y), 2e-4
        moved = np.abs(_np(lp) - want).max()
        most = 2 * bar * np.linalg.norm(Y, axis=1).max() * np.linalg.norm(W, axis=0).max()
        log(f"[step] D={D} rows {err:.1e} (bar {bar:.0e}), log-probabilities {moved:.1e} (bar {most:.1e})")
        assert err <= bar and moved <= most


def test_training_step_in_32_bits():
    """Gradients of a loss of log-probabilities and entropies through the head, the Relation and the norms of its heads
    by the oracles' formulas, and by differences of the 64-bit loss in two directions.

    Bar: evidence to 8 here, fp32 steps of 2^-20 of it forward and backward, some ten terms: 1e-4 of each gradient."""
    rng = np.random.default_rng(8)
    B, H, T, D, V = 2, 2, 70, 32, 300
    mk = lambda *s, std=1.0: torch.from_numpy(rng.standard_normal(s) * std).float().to(DEV).requires_grad_()
    q, k, v = mk(B, H, T, D), mk(B, H, T, D), mk(B, H, T, D)
    wq, wk = (torch.from_numpy(rng.uniform(0.5, 1.4, D)).float().to(DEV).requires_grad_() for _ in range(2))
    head = mk(H * D, V, std=0.3)
    lam = torch.tensor(0.4, device=DEV)
    tokens = torch.from_numpy(rng.integers(0, V, B * T)).to(DEV)
    tokens[::7] = -1
    gl, gh = (torch.from_numpy(rng.standard_normal(B * T)).float().to(DEV) for _ in range(2))
    a, b = R.relation_qk_norm(q, k, wq, wk)
    o = R.relation(a, b, v, lam)
    lp, ent = R.relation_token_logprobs(o.transpose(1, 2).reshape(B * T, H * D) @ head, tokens)
    ((lp * gl).sum() + (ent * gh).sum()).backward()
    torch.cuda.synchronize()

    X = {n: _np(t) for n, t in (("q", q), ("k", k), ("v", v), ("wq", wq), ("wk", wk), ("head", head))}
    pos, L = np.tile(np.arange(T), (B, 1)), float(lam)
    rows = lambda y: y.transpose(0, 2, 1, 3).reshape(B * T, H * D)
    tk, GL, GH = tokens.cpu().numpy(), _np(gl), _np(gh)

    def loss(z):
        y = rows(RO.forward_batched(TO.norm_rope(z["q"], z["wq"], pos), TO.norm_rope(z["k"], z["wk"], pos), z["v"], L)["Y"])
        rs = [TO.logprobs(r, int(t)) for r, t in zip(y @ z["head"], tk)]
        return sum(g * r["logprob"] + h * r["entropy"] for g, h, r in zip(GL, GH, rs)), y
    _, y = loss(X)
    dx = np.stack([TO.logprobs_backward(r, int(t), g, h) for r, t, g, h in zip(y @ X["head"], tk, GL, GH)])
    dy = (dx @ X["head"].T).reshape(B, T, H, D).transpose(0, 2, 1, 3)
    qn, kn = TO.norm_rope(X["q"], X["wq"], pos), TO.norm_rope(X["k"], X["wk"], pos)
    g = RO.backward_batched(qn, kn, X["v"], L, dy)
    want = {"v": g["dv"], "head": y.T @ dx}
    want["q"], want["wq"] = TO.norm_rope_backward(X["q"], X["wq"], pos, g["dq"])
    want["k"], want["wk"] = TO.norm_rope_backward(X["k"], X["wk"], pos, g["dk"])
    for n, t in (("q", q), ("k", k), ("v", v), ("wq", wq), ("wk", wk), ("head", head)):
        err = rel_l2(_np(t.grad), want[n])
        log(f"[training step] d{n}: {err:.1e}")
        assert err <= 1e-4, n
    for seed in range(2):  # error of the difference: h^2 times the third derivative's share, some 1e-6
        way = {n: np.random.default_rng(seed).standard_normal(x.shape) for n, x in X.items()}
        h = 1e-5
        diff = (loss({n: X[n] + h * way[n] for n in X})[0] - loss({n: X[n] - h * way[n] for n in X})[0]) / (2 * h)
        got = sum(float((_np(t.grad) * way[n]).sum()) for n, t in (("q", q), ("k", k), ("v", v), ("wq", wq), ("wk", wk), ("head", head)))
        size = math.sqrt(sum(float((want[n] ** 2).sum()) for n in X))  # of the derivative along such a direction
        assert abs(got - diff) <= 1e-3 * size, (got, diff)


def test_captured_training_step():
    """Norms, Relation and log-probabilities with their backward passes in a graph: the eager gradients' bits on every
    replay; refused while an eager graph of the same leaves lives."""
    rng = np.random.default_rng(30)
    B, H, T, D = 2, 2, 100, 64
    mk = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(torch.bfloat16).to(DEV)
    q, k, wq, z = mk(B, H, T, D), mk(B, H, T, D), mk(D).float(), mk(60, 500)
    tokens = torch.from_numpy(rng.integers(-1, 500, 60)).to(DEV)
    leaves = [t.requires_grad_() for t in (q, k, wq, z)]
    v, lam, c = mk(B, H, T, D), torch.full((), 0.3, device=DEV), mk(B, H, T, D)

    def loss():
        a, b = R.relation_qk_norm(q, k, wq, None)
        lp, ent = R.relation_token_logprobs(z, tokens)
        return (R.relation(a, b, v, lam) * c).float().sum() + (lp * 0.5).sum() + (ent * 0.1).sum()

    def step():
        return torch.autograd.grad(loss(), leaves)
    live = loss()
    for call in (lambda: R.relation_qk_norm(q, k, wq, None), lambda: R.relation_token_logprobs(z, tokens)):
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(RuntimeError, match="lives"):
            with torch.cuda.graph(graph):
                call()
        with torch.no_grad():  # nothing to differentiate, nothing to refuse
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call()
    del live
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for turn in range(4):
        with torch.no_grad():
            for t in leaves:
                t.mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        held = [t.clone() for t in got]
        want = step()
        torch.cuda.synchronize()
        for x, y in zip(held, want):
            assert torch.equal(x, y), turn


def test_captured_steps_that_share_their_workspaces():
    """Two graphs of a step over the same caches and workspaces, replayed in turn with eager work between: the eager
    step's bits."""
    rng = np.random.default_rng(21)
    H, D, page, V, B = 2, 64, 16, 4000, 3
    mk = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(torch.bfloat16).to(DEV)
    W = 320
    table = _i32(rng.permutation(B * W + 4)[:B * W].reshape(B, W))
    kc, vc = mk(B * W + 4, H, page, D), mk(B * W + 4, H, page, D)
    head = mk(H * D, V)
    wq, wk = mk(D), mk(D)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    lam = torch.full((1,), 0.4, device=DEV)

    class Step:
        def __init__(self, added):
            self.added, self.N = added, sum(added)
            self.x, self.tokens = mk(self.N, 3, H, D), torch.from_numpy(rng.integers(0, V, self.N)).to(DEV)
            self.lens, self.start = _i32([5000, 4000, 100]), _i32(np.concatenate([[0], np.cumsum(added)]))
            self.where()

        def where(self):
            n = np.array(self.added)
            first = self.lens.cpu().numpy() - n
            pos = np.concatenate([f + np.arange(c) for f, c in zip(first, n)])
            t, who = table.cpu().numpy(), np.repeat(np.arange(B), n)
            self.pos = _i32(pos) if not hasattr(self, "pos") else self.pos.copy_(_i32(pos))
            slots = torch.from_numpy(t[who, pos // page].astype(np.int64) * page + pos % page).to(DEV)
            self.slots = slots if not hasattr(self, "slots") else self.slots.copy_(slots)

        def run(self):
            q, k, v = self.x.unbind(1)
            f = R.relation_qk_norm_fwd(q, k, wq, wk, self.pos)
            qp = R.relation_paged_append(f["k"], v, kc, vc, self.slots, self.pos, q=f["q"], rope_base=None)
            o = R.relation_paged_prefill(qp, kc, vc, table, self.lens, self.start, lam, workspace=ws)
            p = R.relation_token_logprobs_fwd(o["o"].view(self.N, -1) @ head, self.tokens, top=4, want_rank=True, workspace=ws)
            return [o["o"], o["row_stat"], p["logprob"], p["entropy"], p["rank"], p["top_tokens"], p["top_logprobs"]]

    steps = [Step([40, 1, 3]), Step([1, 1, 60])]
    graphs, outs = [], []
    for s in steps:
        s.run()  # the library product's own first call
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
    for turn in range(4):
        for s in steps:
            s.x.copy_(mk(*s.x.shape))
            s.lens += 1
            s.where()
        before = kc.clone(), vc.clone()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got = [[t.clone() for t in o] for o in outs]
        kc.copy_(before[0])  # each step's rows are in the other's history
        vc.copy_(before[1])
        want = [s.run() for s in steps]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            for x, y in zip(a, b):
                assert torch.equal(x, y), turn


def _prompts(model, lens):
    g = torch.Generator(device=DEV).manual_seed(7)
    return [torch.randint(0, model.emb.shape[0], (n,), device=DEV, generator=g) for n in lens]


@pytest.mark.parametrize("chunk,head_norm,width", [(None, True, 64), (64, False, 64), (17, True, 60), (1, True, 36)])
def test_example_with_chunks_and_norms(chunk, head_norm, width):
    model = E.Decoder(vocab=3001, layers=2, heads=4, width=width, head_norm=head_norm)
    prompts = _prompts(model, (1, 15, 33, 90 if chunk == 1 else 290))
    scores = []
    tokens, _, x = E.generate(model, prompts, 12, chunk=chunk, scores=scores, temperature=0.8, top_k=50)
    torch.cuda.synchronize()
    err = E.check(model, prompts, tokens, x)
    log(f"[example] chunk {chunk} norm {head_norm} width {width}: relative 2-norm {err:.2e} (bar {BAR:.2e})")
    assert err <= BAR
    assert [len(a) for a, _ in scores] == [len(p) - 1 for p in prompts]


def test_example_chunks_have_tokens():
    model = E.Decoder(vocab=301, layers=1, heads=2, width=32)
    for chunk in (0, -1):
        with pytest.raises(ValueError, match="chunk"):
            E.generate(model, _prompts(model, (3,)), 1, chunk=chunk)


def test_example_scores_are_the_prompts_own():
    """Log-probabilities to 1e-5 and ranks by the definition from the same logits."""
    model = E.Decoder(vocab=3001, layers=2, heads=4, width=64, head_norm=True)
    prompts = _prompts(model, (2, 40))
    rows = [model.whole(p) for p in prompts]
    for p, r, (lp, rank) in zip(prompts, rows, E.score(model, prompts, rows)):
        z = (torch.cat(rows) @ model.head)  # one product, as the score has it
        z = z[:len(prompts[0])] if p is prompts[0] else z[len(prompts[0]):]
        for n in range(len(p) - 1):
            w = TO.logprobs(_np(z[n]), int(p[n + 1]))
            assert abs(float(lp[n]) - w["logprob"]) <= 1e-5 * (1 + abs(w["logprob"])) and int(rank[n]) == w["rank"]


def test_prefill_rows_of_no_request_are_left_where_histories_are_split():
    """Rows before, between and behind the requests, and starts that do not ascend, with several slices."""
    rng = np.random.default_rng(4)
    H, D, page, W = 2, 64, 16, 320
    mk = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(torch.bfloat16).to(DEV)
    kc, vc, q = mk(2 * W, H, page, D), mk(2 * W, H, page, D), mk(40, H, D)
    table = _i32(rng.permutation(2 * W).reshape(2, W))
    c, d = R.make_pages(kc, vc), R.RelPagedChunk(40, 2, H, W, 0, 2.0, 0.0)
    assert R.load_library().relation_paged_prefill_workspace_bytes(R.ctypes.byref(c), R.ctypes.byref(d)) > 0
    room = torch.empty((60, H, D), dtype=torch.bfloat16, device=DEV)
    stat = torch.empty((60, H), device=DEV)
    first = R.relation_paged_prefill(q[5:25].contiguous(), kc, vc, table, _i32([5000, 3000]), _i32([0, 8, 20]), 0.4)
    for start, rows in (([5, 13, 25], slice(5, 25)), ([30, 20, 10], None), ([-9, 10 ** 9, 3], None), ([40, 40, 40], slice(0, 0))):
        room.fill_(7.0)
        stat.fill_(7.0)
        R.relation_paged_prefill(q, kc, vc, table, _i32([5000, 3000]), _i32(start), 0.4,
                                 out={"o": room[10:50], "row_stat": stat[10:50]})
        torch.cuda.synchronize()
        assert bool((room[:10] == 7).all()) and bool((room[50:] == 7).all()) and bool((stat[:10] == 7).all()) and bool((stat[50:] == 7).all())
        if rows is not None:
            left = torch.ones(40, dtype=torch.bool, device=DEV)
            left[rows] = False
            assert bool((room[10:50][left] == 7).all()) and bool((stat[10:50][left] == 7).all())
            if rows.stop > rows.start:
                assert rel_l2(_np(room[10:50][rows]), _np(first["o"])) <= 2.0 ** -7 and torch.isfinite(stat[10:50][rows]).all()
