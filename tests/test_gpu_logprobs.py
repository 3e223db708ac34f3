"""GPU parity of the log-probabilities of given tokens, entropy, rank, top alternatives and their gradient with the fp64
oracle.

Bars. Whole numbers are equal. Log-probabilities and entropy: an exponent of up to some 40 rounded to fp32 (4e-6 of a
weight), so 1e-5 absolute and of the value. Gradient, per element: half a step of the type (bf16 2^-8, fp32 2^-24) of
the value; the exponent's fp32 steps, 2^-22 (2 + |log p|) of each product with p, the entropy's 1e-5 of its own; 2^-23
of g at the given token; and what underflows, 2^-120."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import token_oracle as TO
from paper_2608_20172_amd import binding as R
from tests.gpu_helpers import TORCH_DT, log

pytestmark = pytest.mark.gpu

DEV = "cuda"
STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    R.load_library()


def _np(t):
    return t.detach().double().cpu().numpy()


def _logits(N, V, dtype, rng, slope=1.2, ranked=False):
    rank = np.arange(V)[None] if ranked else rng.random((N, V)) * V
    return torch.from_numpy(-slope * np.log1p(rank) + 0.3 * rng.standard_normal((N, V))).to(TORCH_DT[dtype]).to(DEV)


def _check(x, tokens, top=0, grad=True, rows=None):
    """x [N, V] on the device; tokens: a list. Returns what the calls gave."""
    N, V = x.shape
    t = torch.tensor(tokens, dtype=torch.int64, device=DEV)
    f = R.relation_token_logprobs_fwd(x, t, top=top, want_rank=True)
    g = torch.linspace(-1.5, 2.0, N, device=DEV) if N > 1 else torch.full((1,), 0.7, device=DEV)
    h = torch.linspace(0.4, -0.3, N, device=DEV) if N > 1 else torch.full((1,), -0.2, device=DEV)
    d = R.relation_token_logprobs_bwd(x, t, f["stats"], g, h) if grad else None
    torch.cuda.synchronize()
    f = {n: v.cpu() for n, v in f.items()}
    worst = {"lp": 0.0, "H": 0.0, "top": 0.0, "d": 0.0}
    dtype = "bf16" if x.dtype == torch.bfloat16 else "f32"
    for n in (range(N) if rows is None else rows):
        row = _np(x[n])
        w = TO.logprobs(row, int(tokens[n]), top)
        assert int(f["rank"][n]) == w["rank"], (n, int(f["rank"][n]), w["rank"])
        assert f["top_tokens"][n].tolist() == w["top_tokens"], (n, f["top_tokens"][n].tolist(), w["top_tokens"])
        pairs = [("lp", float(f["logprob"][n]), w["logprob"]), ("H", float(f["entropy"][n]), w["entropy"])]
        pairs += [("top", a, b) for a, b in zip(f["top_logprobs"][n].tolist(), w["top_logprobs"])]
        for k, a, b in pairs:
            with np.errstate(over="ignore"):
                b = float(np.float32(b))  # the lowest number below the largest: -2^129, which fp32 has as -inf
            if not math.isfinite(b):
                assert a == b or (math.isnan(a) and math.isnan(b)), (n, k, a, b)
            else:
                worst[k] = max(worst[k], abs(a - b) / (1e-5 * (1 + abs(b))))
        if grad:
            gn, hn = float(g[n]), float(h[n])
            want, got = TO.logprobs_backward(row, int(tokens[n]), gn, hn), _np(d[n])
            assert np.array_equal(np.isnan(want), np.isnan(got)), n
            if np.isnan(want).any():
                continue
            p, lp = w["p"], np.where(w["p"] > 0, w["logp"], 0.0)
            size = abs(gn) * (tokens[n] >= 0) + abs(hn) * (np.abs(lp) + w["entropy"])
            bar = STEP[dtype] * np.abs(want) + 2.0 ** -22 * (2 + np.abs(lp)) * p * size + \
                1e-5 * p * abs(hn) * (1 + w["entropy"]) + 2.0 ** -120
            if tokens[n] >= 0:
                bar[tokens[n]] += 2.0 ** -23 * abs(gn)
            worst["d"] = max(worst["d"], float(np.max(np.abs(got - want) / bar)))
    log("  " + ", ".join(f"{k} {v:.2f}" for k, v in worst.items()) + " of the bars")
    assert max(worst.values()) <= 1.0, worst
    return f, d


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,V,top", [
    (1, 1, 1), (1, 2, 0), (3, 3, 3), (2, 7, 5), (2, 8, 8), (3, 9, 9), (2, 33, 32), (5, 255, 20), (2, 1023, 1), (2, 1025, 32),
    (3, 2047, 5), (2, 2049, 20), (2, 4099, 20), (2, 8192, 20), (2, 8193, 8), (2, 16385, 32), (3, 32000, 5), (2, 50257, 20),
    (1, 131072, 32), (2, 65537, 0), (40, 5003, 4),
])
def test_rows(N, V, top, dtype):
    rng = np.random.default_rng(V + N)
    log(f"[logprobs] {N} x {V} top {top} {dtype}")
    for ranked in (False, True):
        x = _logits(N, V, dtype, rng, ranked=ranked)
        best = x.float().argmax(1).tolist()
        tokens = [best[n] if n % 2 == 0 else int(rng.integers(V)) for n in range(N)]
        _check(x, tokens, top)
    _check(x, [0 if n % 2 else V - 1 for n in range(N)], top, grad=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_very_long_rows(dtype):
    """2^22 logits: several sub-chunks a workgroup, with alternatives and without."""
    rng = np.random.default_rng(9)
    x = _logits(1, 1 << 22, dtype, rng)
    for top in (0, 5, 32):
        _check(x, [int(rng.integers(1 << 22))], top, grad=top == 0)
    x = _logits(1, (1 << 22) - 5, dtype, rng, ranked=True).flip(1)  # the likeliest at the very end
    _check(x.contiguous(), [(1 << 22) - 6], 32, grad=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [40, 3000, 9000, 40000])
def test_ties(V, dtype):
    """All equal, two values, few values, a flat row with one above, zeros of both signs: the lowest indices first."""
    rng = np.random.default_rng(V)
    rows = [np.full(V, 1.5), rng.integers(0, 2, V), rng.integers(0, 9, V) / 4.0, np.zeros(V), np.where(rng.random(V) < 0.5, 0.0, -0.0),
            np.where(rng.random(V) < 0.5, 0.0, -0.0) - (np.arange(V) % 3 == 0), np.full(V, -3.0)]
    rows[3][V - 2] = 2.0
    x = torch.from_numpy(np.stack(rows)).to(TORCH_DT[dtype]).to(DEV)
    for tokens in ([V - 1] * 7, [0] * 7, [V // 2] * 7, [V - 2] * 7, [int(t) for t in rng.integers(0, V, 7)]):
        for top in (1, 20, 32):
            _check(x, tokens, top, grad=top == 1)


@pytest.mark.parametrize("V", [5, 300, 9001, 33000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masked_infinite_and_nan_logits(V, dtype):
    """-inf (all but a few, all), the type's lowest value, +inf (one, several, all), NaN, large values, and tokens that
    are masked, absent or out of range."""
    rng = np.random.default_rng(V)
    lowest = float(torch.finfo(TORCH_DT[dtype]).min)
    top = min(V, 20)
    base = rng.standard_normal(V)
    rows = []
    for kind in range(12):
        r = base.copy()
        some = rng.choice(V, 3, replace=False)
        if kind == 0: r[:] = -np.inf; r[some] = base[some]
        if kind == 1: r[:] = -np.inf
        if kind == 2: r[:] = lowest; r[some] = base[some]
        if kind == 3: r[:] = lowest
        if kind == 4: r[some[0]] = np.inf
        if kind == 5: r[some] = np.inf
        if kind == 6: r[:] = np.inf
        if kind == 7: r[some] = np.nan
        if kind == 8: r[:] = np.nan
        if kind == 9: r[:] = np.nan; r[some[0]] = 1.0; r[some[1]] = -np.inf
        if kind == 10: r *= 1.0e30
        if kind == 11: r[some[0]] = -lowest; r[some[1]] = lowest
        rows.append(r)
    x = torch.from_numpy(np.stack(rows)).to(TORCH_DT[dtype]).to(DEV)
    best = torch.nan_to_num(x.float(), nan=-math.inf, posinf=3.0e38, neginf=-3.0e38).argmax(1).tolist()
    for tokens in (best, [0] * 12, [V - 1] * 12, [-1] * 12, [V] * 12, [int(t) for t in rng.integers(0, V, 12)]):
        _check(x, tokens, top)
    # signalling NaN patterns count as -inf as well
    bits = torch.int16 if dtype == "bf16" else torch.int32
    y = x[:2].clone()
    y[0] = torch.from_numpy(base).to(y.dtype).to(DEV)
    y[0].view(bits)[1] = 0x7F81 if dtype == "bf16" else 0x7F800001
    _check(y[:1], [0], top)


def test_negative_and_far_tokens():
    x = _logits(6, 500, "f32", np.random.default_rng(2))
    t = torch.tensor([-1, -2 ** 62, 500, 2 ** 33 + 3, 2 ** 62, 3], device=DEV)
    f = R.relation_token_logprobs_fwd(x, t, want_rank=True)
    assert f["logprob"][:2].tolist() == [0.0, 0.0] and torch.isnan(f["logprob"][2:5]).all() and f["rank"][:5].tolist() == [-1] * 5
    d = R.relation_token_logprobs_bwd(x, t, f["stats"], torch.ones(6, device=DEV), None)
    assert not d[:2].any() and torch.isnan(d[2:5]).all() and torch.isfinite(d[5]).all()
    d = R.relation_token_logprobs_bwd(x, t, f["stats"], None, torch.ones(6, device=DEV))
    e = R.relation_token_logprobs_bwd(x, torch.full_like(t, 3), f["stats"], None, torch.ones(6, device=DEV))
    assert torch.equal(d[:2], e[:2]) and torch.equal(d[5], e[5])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_alignment(dtype):
    rng = np.random.default_rng(5)
    big = _logits(7, 3333, dtype, rng)
    t = torch.tensor([5, 0, 3000, 77, -1, 3000, 9], device=DEV)
    g, h = torch.randn(7, device=DEV), torch.randn(7, device=DEV)
    for view in (big[:, 1:3002], big[::2, 3:3004], big[:, ::2], big[:1].expand(7, 3333), big.t().contiguous().t()):
        n = view.shape[0]
        a = R.relation_token_logprobs_fwd(view, t[:n].clamp(max=1600), top=7, want_rank=True)
        b = R.relation_token_logprobs_fwd(view.contiguous(), t[:n].clamp(max=1600), top=7, want_rank=True)
        assert all(torch.equal(a[k], b[k]) for k in a)
        da = R.relation_token_logprobs_bwd(view, t[:n].clamp(max=1600), a["stats"], g[:n], h[:n])
        guard = torch.full((n, view.shape[1] + 9), 7.0, dtype=view.dtype, device=DEV)
        db = R.relation_token_logprobs_bwd(view.contiguous(), t[:n].clamp(max=1600), b["stats"], g[:n], h[:n],
                                           out={"dlogits": guard[:, 4:-5]})
        assert torch.equal(da, db) and bool((guard[:, :4] == 7).all()) and bool((guard[:, -5:] == 7).all())


def test_offsets_past_32_bits():
    """2^32 logits and more: the last rows."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 20 GB")
    N, V = 33000, 131072
    x = torch.zeros((N, V), dtype=torch.bfloat16, device=DEV)
    x[-2:] = _logits(2, V, "bf16", np.random.default_rng(6))
    t = torch.full((N,), 17, device=DEV)
    f = R.relation_token_logprobs_fwd(x, t, top=3, want_rank=True)
    want = R.relation_token_logprobs_fwd(x[-2:].clone(), t[-2:], top=3, want_rank=True)
    assert all(torch.equal(f[k][-2:], want[k]) for k in f) and f["rank"][:-2].unique().tolist() == [17]
    g = torch.ones(N, device=DEV)
    d = R.relation_token_logprobs_bwd(x, t, f["stats"], g, g)
    e = R.relation_token_logprobs_bwd(x[-2:].clone(), t[-2:], want["stats"], g[-2:], g[-2:])
    assert torch.equal(d[-2:], e)
    del x, d
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [3, 5000])
def test_rows_without_a_token_count_for_nothing(V, dtype):
    """Padding rows, whatever stands there: logprob 0, and a gradient of 0 unless the entropy is asked for."""
    x = _logits(6, V, dtype, np.random.default_rng(3))
    x[1], x[2], x[3] = math.nan, -math.inf, math.inf
    t = torch.tensor([2, -1, -1, -1, -5, 0], device=DEV)
    leaf = x.clone().requires_grad_()
    lp, H = R.relation_token_logprobs(leaf, t)
    assert lp[1:5].tolist() == [0.0] * 4 and torch.isfinite(lp).all()
    (lp.sum() + torch.where(t >= 0, H, 0.0).sum()).backward()
    assert not leaf.grad[1:5].any() and torch.isfinite(leaf.grad).all() and leaf.grad[0].any() and leaf.grad[5].any()
    f = R.relation_token_logprobs_fwd(x, t)
    g, h = torch.full((6,), math.inf, device=DEV), torch.tensor([0.0, 0.0, 0.0, 0.0, 0.5, 0.0], device=DEV)
    d = R.relation_token_logprobs_bwd(x, t, f["stats"], g, h)
    assert not d[1:4].any() and d[4].any() and torch.isfinite(d[4]).all()


def test_gradient_of_more_threads_than_a_grid_has():
    """2^34 gradients in fp32, four a thread: rows of every part of the grid."""
    N, V = 131200, 131072
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 69 GB")
    x = _logits(1, V, "f32", np.random.default_rng(4))
    t = torch.full((N,), 7, device=DEV)
    f = R.relation_token_logprobs_fwd(x, t[:1])
    stats, g, h = f["stats"].expand(N, 4).contiguous(), torch.ones(N, device=DEV), torch.ones(N, device=DEV)
    d = torch.empty((N, V), device=DEV)
    R.relation_token_logprobs_bwd(x.expand(N, V), t, stats, g, h, out={"dlogits": d})
    want = R.relation_token_logprobs_bwd(x, t[:1], stats[:1], g[:1], h[:1])[0]
    for n in (0, 1, 65535, 65536, 131070, 131071, 131072, 131198, 131199):
        assert torch.equal(d[n], want), n
    del d
    torch.cuda.empty_cache()


def test_gradients_by_differences_and_through_autograd():
    """Central differences of the forward kernel in fp32 along random directions, step 2^-6: the cubic term is some
    1e-4 of the gradient's size, the rounding of the outputs 1e-5; bar 2e-3."""
    rng = np.random.default_rng(8)
    x = _logits(9, 700, "f32", rng)
    t = torch.tensor([3, 0, 699, -1, 5, 5, 100, -7, 1], device=DEV)
    g, h = torch.randn(9, device=DEV), torch.randn(9, device=DEV)
    leaf = x.clone().requires_grad_()
    lp, H = R.relation_token_logprobs(leaf, t)
    (d,) = torch.autograd.grad((lp * g).sum() + (H * h).sum(), leaf)

    def f(x):
        r = R.relation_token_logprobs_fwd(x, t)
        return float((r["logprob"].double() * g).sum() + (r["entropy"].double() * h).sum())
    for _ in range(4):
        u, e = torch.randn(x.shape, device=DEV), 2.0 ** -6
        num, ana = (f(x + e * u) - f(x - e * u)) / (2 * e), float((d.double() * u).sum())
        assert abs(num - ana) <= 2e-3 * float(d.norm()), (num, ana)
    # one of the two alone, shared rows, and the plain definition's own gradient
    for pick in (0, 1):
        a, b = x.clone().requires_grad_(), x.double().requires_grad_()
        R.relation_token_logprobs(a, t)[pick].sum().backward()
        logp = torch.log_softmax(b, 1)
        ref = (torch.where(t < 0, 0.0, logp.gather(1, t.clamp(min=0)[:, None])[:, 0]), -(logp.exp() * logp).sum(1))[pick]
        ref.sum().backward()
        assert float((a.grad - b.grad).abs().max()) <= 1e-6
    row = x[:1].clone().requires_grad_()
    R.relation_token_logprobs(row.expand(9, 700), t)[0].sum().backward()
    assert row.grad.shape == (1, 700) and torch.isfinite(row.grad).all()


def test_repeats_its_bits_on_a_stream_and_in_a_graph():
    x = _logits(50, 40000, "bf16", np.random.default_rng(11))
    x[3] = 1.0  # a flat row
    t = torch.randint(0, 40000, (50,), device=DEV)
    g = torch.randn(50, device=DEV)

    def step():
        f = R.relation_token_logprobs_fwd(x, t, top=20, want_rank=True)
        return [f[k] for k in sorted(f)] + [R.relation_token_logprobs_bwd(x, t, f["stats"], g, g)]
    first = step()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = step()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for turn in range(3):
        x.mul_(1.25)
        t.add_(7).remainder_(40000)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))


def test_it_agrees_with_the_sampler():
    """The sampled token's log-probability at temperature 1."""
    x = _logits(20, 32000, "f32", np.random.default_rng(12))
    s = R.relation_sample(x, torch.empty_like(x).exponential_())
    f = R.relation_token_logprobs_fwd(x, s["tokens"])
    assert float((f["logprob"] - s["logprob"]).abs().max()) <= 2e-5 * (1 + float(s["logprob"].abs().max()))


def test_given_outputs_and_arguments():
    x = _logits(4, 100, "f32", np.random.default_rng(13))
    t = torch.tensor([1, 2, 3, 4], device=DEV)
    out = {"logprob": torch.empty(4, device=DEV), "top_tokens": torch.empty((4, 2), dtype=torch.int64, device=DEV)}
    f = R.relation_token_logprobs_fwd(x, t.int(), top=2, out=out)
    assert f["logprob"] is out["logprob"] and f["top_tokens"] is out["top_tokens"] and f["rank"] is None
    for bad in (dict(top=33), dict(top=-1)):
        with pytest.raises(RuntimeError):
            R.relation_token_logprobs_fwd(x, t, **bad)
    with pytest.raises(RuntimeError, match="alternatives"):
        R.relation_token_logprobs_fwd(x[:, :5], t, top=6)
    for a in ((x[0], t), (x, t[:3]), (x, t.float()), (x.cpu(), t), (x.half(), t)):
        with pytest.raises((ValueError, TypeError)):
            R.relation_token_logprobs_fwd(*a)
    for a in ((f["stats"][:3],), (f["stats"], t[:3].float()), (f["stats"].double(),)):
        with pytest.raises(ValueError):
            R.relation_token_logprobs_bwd(x, t, *a)
    with pytest.raises(ValueError):
        R.relation_token_logprobs_fwd(x, t, out={"logprob": torch.empty(5, device=DEV)})
    e = R.relation_token_logprobs_fwd(x[:0], t[:0], top=3)
    assert e["logprob"].shape == (0,) and R.relation_token_logprobs_bwd(x[:0], t[:0], e["stats"]).shape == (0, 100)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,left", [(260, 4), (261, 5), (263, 7), (300, 3), (515, 3), (516, 4), (517, 1), (772, 4), (2050, 2),
                                    (4099, 3), (30981, 5), (61445, 5)])
def test_rows_masked_everywhere_but_at_the_end(V, left, dtype):
    """A mask of a finite value under -2^119 on all but the last logits: the alternatives past those are masked tokens, the
    lowest indices first, each once."""
    rng = np.random.default_rng(V)
    lowest = float(torch.finfo(TORCH_DT[dtype]).min)
    rows = np.stack([np.full(V, x) for x in (lowest, -1.0e38, lowest, -7.0e35, -6.0e35, -1.0e30)])
    rows[:, V - left:] = rng.standard_normal((len(rows), left))
    rows[2, 1] = 0.5  # one at the front as well
    x = torch.from_numpy(rows).to(TORCH_DT[dtype]).to(DEV)
    n = len(rows)
    for top in (1, left, left + 1, 8, 20, 32):
        _check(x, [V - 1] * n, top, grad=False)
    _check(x, [0, V - left, 1, V - 2, 3, V // 2], 20)


@pytest.mark.parametrize("dtype,V", [("f32", 30981), ("f32", 31743), ("bf16", 61445), ("bf16", 63487)])
def test_many_rows_masked_everywhere_but_at_the_end(V, dtype):
    """The same in a workgroup's last of several sub-chunks, when all before it are masked."""
    N, left = 600, V % 1024 if V % 1024 < 8 else 5
    x = torch.full((N, V), float(torch.finfo(TORCH_DT[dtype]).min), dtype=TORCH_DT[dtype], device=DEV)
    x[:, V - left:] = torch.from_numpy(np.random.default_rng(V).standard_normal((N, left))).to(x)
    for top in (left, left + 1, 20, 32):
        _check(x, [V - 1 - n % 3 for n in range(N)], top, grad=False, rows=[0, 1, 300, 599])


def test_outputs_are_worked_on_in_place():
    """Log-probabilities and entropies masked and scaled in place, as a loss is: gradients by the formula's own in 64
    bits. Exponents under 10 leave 1e-6 of a weight and of Z, 2e-6 of p, 4e-6 of the entropy: 0.5 * 2e-6 + 0.25 * (10 * 2e-6 +
    4e-6) at most, bar 1e-5."""
    rng = np.random.default_rng(17)
    x = _logits(8, 300, "f32", rng)
    t = torch.from_numpy(rng.integers(0, 300, 8)).to(DEV)
    mask = torch.tensor([0, 1, 0, 0, 1, 0, 1, 0], dtype=torch.bool, device=DEV)

    def loss(lp, ent):
        lp.masked_fill_(mask, 0.0)
        lp *= 0.5
        ent[0] = 0.0
        ent.mul_(0.25)
        return lp.sum() + ent.sum()
    a, b = x.clone().requires_grad_(), x.double().requires_grad_()
    loss(*R.relation_token_logprobs(a, t)).backward()
    logp = torch.log_softmax(b, 1)
    loss(logp.gather(1, t[:, None])[:, 0], -(logp.exp() * logp).sum(1)).backward()
    assert float((a.grad - b.grad).abs().max()) <= 1e-5
    # numbers that were written over outside the graph are not what the backward pass reads
    c = x.clone().requires_grad_()
    lp, ent = R.relation_token_logprobs(c, t)
    want = torch.autograd.grad(lp.sum() + ent.sum(), c, retain_graph=True)[0]
    lp.detach().mul_(3.0)
    ent.detach().zero_()
    assert torch.equal(torch.autograd.grad(lp.sum() + ent.sum(), c)[0], want)
    # an output kept for later keeps only itself
    for o in R.relation_token_logprobs(x, t):
        assert o.untyped_storage().nbytes() == 8 * 4
    f = R.relation_token_logprobs_fwd(x, t, top=3)
    stats = f["stats"]._version
    f["logprob"].zero_()
    f["top_logprobs"].zero_()
    assert stats == f["stats"]._version
