"""GPU parity of the norms of query and key heads with the position rotation, forward and backward, with the fp64 oracle.

Bars, per element: half a step of the type (bf16 2^-8, fp32 2^-24, of the value) for the one rounding of an output, and
2^-20 (backward: 2^-19, twice the steps) of what it is made of for the fp32 arithmetic: a sum of up to 128 squares,
the root, sine and cosine, each some 2^-23. Weights' gradients: 2^-17 of the sum of their terms' sizes (at most some
hundred fp32 additions one after another)."""
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


def _reference(x, w, pos, dy=None, *, norm=True, eps=1.0e-6, rope_dim=None, layout="half", amplitude=1.0, **kw):
    """The oracle's definitions over whole tensors in 64 bits (test_reference holds them together): y and what its
    elements are made of; with dy: dx, what it is made of, dw and the sum of its terms' sizes."""
    x = x.double()
    B, H, T, D = x.shape
    d = D if rope_dim is None else rope_dim
    w = torch.ones(D, dtype=torch.float64, device=DEV) if w is None else w.double()
    pos = torch.arange(T, device=DEV).expand(B, T) if pos is None else pos.expand(B, T)
    live = (pos >= 0)[:, None, :, None]
    ang = pos.double()[:, None, :, None] * torch.tensor(TO.frequencies(d, **kw), dtype=torch.float64, device=DEV)
    cs, sn = torch.cos(ang) * amplitude, torch.sin(ang) * amplitude

    def turned(z, s):
        z = z.clone()
        a, b = (z[..., 0:d:2].clone(), z[..., 1:d:2].clone()) if layout == "interleaved" else (z[..., :d // 2].clone(), z[..., d // 2:d].clone())
        p, q = a * cs - b * s, a * s + b * cs
        if layout == "interleaved":
            z[..., 0:d:2], z[..., 1:d:2] = p, q
        else:
            z[..., :d // 2], z[..., d // 2:d] = p, q
        return z
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) if norm else torch.ones_like(x[..., :1])
    amp = max(1.0, abs(amplitude)) * 2
    if dy is None:
        n = x * r * w
        return torch.where(live, turned(n, sn), 0.0), torch.where(live, n.abs().amax(-1, keepdim=True) * amp, 0.0)
    g = turned(dy.double(), -sn)
    if not norm:
        return torch.where(live, g, 0.0), torch.where(live, g.abs().amax(-1, keepdim=True) * 2 + dy.double().abs().amax(-1, keepdim=True) * amp, 0.0), None, None
    xr, gw = x * r, g * w
    dx = r * (gw - xr * (gw * xr).mean(-1, keepdim=True))
    size = dy.double().abs().amax(-1, keepdim=True) * amp * w.abs().max()
    parts = r * size * (1 + xr.abs().amax(-1, keepdim=True) * xr.abs().mean(-1, keepdim=True))
    terms = torch.where(live, g * xr, 0.0)
    big = torch.where(live, xr.abs() * dy.double().abs().amax(-1, keepdim=True) * amp, 0.0)
    return torch.where(live, dx, 0.0), torch.where(live, parts, 0.0), terms.sum((0, 1, 2)), big.sum((0, 1, 2))


def test_reference():
    """The whole-tensor reference is the oracle."""
    g = torch.Generator(device=DEV).manual_seed(1)
    x, dy = (torch.randn(2, 3, 4, 12, device=DEV, generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.rand(12, device=DEV, generator=g, dtype=torch.float64) + 0.5
    pos = torch.tensor([[0, 1, 70000, -2], [5, 5, 9, 1 << 20]], device=DEV)
    for kw in (dict(), dict(layout="interleaved", rope_dim=8, amplitude=1.2), dict(norm=False, rope_dim=6),
               dict(factor=4.0, original_length=128), dict(rope_dim=0), dict(factor=2.0, low=2.0, high=5.0, original_length=99)):
        ww = w if kw.get("norm", True) else None
        wn = None if ww is None else _np(ww)
        assert np.allclose(_np(_reference(x, ww, pos, **kw)[0]), TO.norm_rope(_np(x), wn, _np(pos), **kw), atol=1e-9)
        dx, dw = TO.norm_rope_backward(_np(x), wn, _np(pos), _np(dy), **kw)
        r = _reference(x, ww, pos, dy, **kw)
        assert np.allclose(_np(r[0]), dx, atol=1e-9)
        assert ww is None or np.allclose(_np(r[2]), dw, atol=1e-8)


def _close(name, got, want, parts, dtype, factor):
    bar = STEP[dtype] * want.abs() + factor * parts
    worst = float(((got.double() - want).abs() / bar.clamp(min=1e-30)).max()) if want.numel() else 0.0
    log(f"  {name}: {worst:.2f} of the bar")
    assert worst <= 1.0, name


def _heads(shape, dtype, place, g):
    """q and k [B, heads, T, D]: slices of a projection, dense, or views with other strides."""
    B, Hq, H, T, D = shape
    t = TORCH_DT[dtype]
    big = lambda *s: (torch.randn(*s, device=DEV, generator=g) * torch.exp(torch.randn(s[:-1] + (1,), device=DEV, generator=g))).to(t)
    if place == "projection":
        x = big(B, T, Hq + 2 * H, D)
        return x[:, :, :Hq].transpose(1, 2), x[:, :, Hq:Hq + H].transpose(1, 2)
    if place == "odd":  # rows on any element, a gap between them
        x = big(B, Hq + H, T, D + 3)
        return x[:, :Hq, :, 1:D + 1], x[:, Hq:, :, 2:D + 2]
    if place == "across":  # batch inside tokens
        x = big(T, B, Hq + H, D).permute(1, 2, 0, 3)
        return x[:, :Hq], x[:, Hq:]
    return big(B, Hq, T, D), big(B, H, T, D)


CASES = [
    # B, Hq, H, T, D, dtype, place, weights, positions, options
    (1, 1, 1, 1, 64, "bf16", "dense", "f32", None, {}),
    (2, 8, 8, 33, 64, "bf16", "projection", "f32", "each", {}),
    (1, 8, 2, 64, 80, "bf16", "projection", "bf16", "each", {}),
    (1, 4, 4, 17, 60, "bf16", "dense", "f32", "shared", {}),
    (2, 12, 12, 100, 64, "f32", "projection", "f32", None, {}),
    (1, 16, 4, 50, 128, "bf16", "projection", "bf16", "each", dict(rope_dim=64, layout="interleaved", factor=8.0, original_length=2048, amplitude=1.2)),
    (3, 2, 1, 9, 128, "f32", "across", "f32", "each", dict(layout="interleaved")),
    (2, 3, 2, 21, 48, "bf16", "odd", None, "each", dict(rope_dim=24)),
    (2, 3, 2, 21, 48, "f32", "odd", "f32", "each", dict(rope_dim=22, layout="interleaved")),
    (1, 2, 3, 13, 6, "bf16", "odd", "f32", "each", dict(rope_dim=2)),
    (1, 2, 2, 5, 63, "bf16", "odd", "bf16", "shared", dict(rope_dim=62)),
    (1, 5, 1, 7, 127, "f32", "dense", "f32", "each", dict(rope_dim=0)),
    (1, 2, 2, 7, 1, "f32", "dense", "f32", None, dict(rope_dim=0)),
    (1, 2, 2, 7, 2, "bf16", "dense", "f32", None, dict(eps=0.5)),
    (2, 2, 2, 40, 64, "bf16", "projection", None, "each", dict(norm=False, layout="interleaved")),
    (2, 2, 2, 40, 96, "f32", "projection", None, "each", dict(norm=False, factor=4.0)),
    (4, 3, 1, 1100, 32, "bf16", "projection", "f32", "each", {}),
    (1, 2, 2, 4096, 64, "bf16", "projection", "f32", "each", {}),
    (5, 2, 1, 1801, 16, "f32", "across", "f32", "each", dict(rope_dim=8)),
    (3, 1, 2, 3003, 8, "bf16", "projection", "bf16", "shared", dict(layout="interleaved")),
    (1, 0, 3, 20, 64, "bf16", "projection", "f32", "each", {}),
    (1, 3, 0, 20, 64, "bf16", "dense", "f32", "each", {}),
]


@pytest.mark.parametrize("B,Hq,H,T,D,dtype,place,weights,positions,kw", CASES)
def test_norm(B, Hq, H, T, D, dtype, place, weights, positions, kw):
    log(f"[qk_norm] B={B} Hq={Hq} H={H} T={T} D={D} {dtype} {place} weights={weights} positions={positions} {kw}")
    g = torch.Generator(device=DEV).manual_seed(B * 1000 + T + D)
    q, k = _heads((B, Hq, H, T, D), dtype, place, g)
    dq, dk = _heads((B, Hq, H, T, D), dtype, "projection" if place == "dense" else "dense", g)
    wq, wk = (None if weights is None else (1 + 0.3 * torch.randn(D, device=DEV, generator=g)).to(TORCH_DT[weights]) for _ in range(2))
    pos = None
    if positions is not None:
        shape = (T,) if positions == "shared" else (B, T)
        pos = torch.randint(0, 1 << 22, shape, device=DEV, generator=g, dtype=torch.int32)
        pos[..., T // 2] = -1 - T  # a token of nobody
    q, k, dq, dk = (x if n else None for x, n in ((q, Hq), (k, H), (dq, Hq), (dk, H)))
    wq, wk = (wq if Hq else None), (wk if H else None)
    y = R.relation_qk_norm_fwd(q, k, wq, wk, pos, **kw)
    d = R.relation_qk_norm_bwd(q, k, wq, wk, dq, dk, pos, **kw)
    torch.cuda.synchronize()
    for n, x, w, gx in (("q", q, wq, dq), ("k", k, wk, dk)):
        if x is None:
            assert y[n] is None and d["d" + n] is None
            continue
        want, parts = _reference(x, w, pos, **kw)
        _close(n, y[n], want, parts, dtype, 2.0 ** -20)
        want, parts, dw, size = _reference(x, w, pos, gx, **kw)
        _close("d" + n, d["d" + n], want, parts, dtype, 2.0 ** -19)
        if w is not None:
            _close("dw" + n, d["dw" + n], dw, size, "f32", 2.0 ** -17)
        else:
            assert d["dw" + n] is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packed_tokens_are_a_batch_of_one(dtype):
    g = torch.Generator(device=DEV).manual_seed(2)
    q, k = (torch.randn(37, h, 80, device=DEV, generator=g).to(TORCH_DT[dtype]) for h in (8, 2))
    w = torch.rand(80, device=DEV, generator=g)
    pos = torch.randint(0, 5000, (37,), device=DEV, generator=g, dtype=torch.int32)
    a = R.relation_qk_norm_fwd(q, k, w, w, pos)
    b = R.relation_qk_norm_fwd(*(x.transpose(0, 1)[None] for x in (q, k)), w, w, pos)
    c = R.relation_qk_norm_fwd(q, k, w, w, pos.long())
    for n in ("q", "k"):
        assert torch.equal(a[n], b[n][0].transpose(0, 1)) and torch.equal(a[n], c[n]) and a[n].is_contiguous()
    da = R.relation_qk_norm_bwd(q, k, w, w, a["q"], a["k"], pos)
    db = R.relation_qk_norm_bwd(*(x.transpose(0, 1)[None] for x in (q, k)), w, w, b["q"], b["k"], pos[None])
    assert torch.equal(da["dq"], db["dq"][0].transpose(0, 1)) and torch.equal(da["dwq"], db["dwq"]) and torch.equal(da["dwk"], db["dwk"])


def test_expanded_inputs_and_given_outputs():
    """Inputs of stride 0 (one head for all, a gradient of ones), outputs as slices of one buffer."""
    g = torch.Generator(device=DEV).manual_seed(3)
    one = torch.randn(2, 1, 9, 64, device=DEV, generator=g).to(torch.bfloat16)
    q, k = one.expand(2, 4, 9, 64), one.expand(2, 2, 9, 64)
    buf = torch.full((2, 9, 8, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    out = {"q": buf[:, :, :4].transpose(1, 2), "k": buf[:, :, 4:6].transpose(1, 2)}
    y = R.relation_qk_norm_fwd(q, k, out=out)
    want = R.relation_qk_norm_fwd(q.contiguous(), k.contiguous())
    assert y["q"] is out["q"] and torch.equal(y["q"], want["q"]) and torch.equal(y["k"], want["k"]) and bool((buf[:, :, 6:] == 7).all())
    ones = torch.ones((), dtype=torch.bfloat16, device=DEV)
    w = torch.ones(64, device=DEV)
    buf.fill_(7.0)
    out = {"dq": buf[:, :, :4].transpose(1, 2), "dk": buf[:, :, 4:6].transpose(1, 2)}
    d = R.relation_qk_norm_bwd(q, k, w, w, ones.expand(q.shape), ones.expand(k.shape), out=out)
    e = R.relation_qk_norm_bwd(q.contiguous(), k.contiguous(), w, w, torch.ones_like(q.contiguous()), torch.ones_like(k.contiguous()))
    assert torch.equal(d["dq"], e["dq"]) and torch.equal(d["dk"], e["dk"]) and torch.equal(d["dwq"], e["dwq"])
    for bad in ({"q": q}, {"q": buf[:, :, :4].transpose(1, 2), "k": buf[:, :, 2:4].transpose(1, 2)}):
        with pytest.raises(RuntimeError, match="overlap"):
            R.relation_qk_norm_fwd(q, k, out=bad)


def test_zeros_infinities_and_nan_stay_in_their_rows():
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(1, 2, 12, 64, device=DEV, generator=g)
    x[0, 0, 3] = 0.0
    base = R.relation_qk_norm_fwd(x, None)["q"]
    assert not base[0, 0, 3].any() and torch.isfinite(base).all()
    z = x.clone()
    z[0, 1, 5, 7], z[0, 0, 6, 0], z[0, 1, 8] = math.nan, math.inf, 1.0e30  # a square past fp32
    y = R.relation_qk_norm_fwd(z, None)["q"]
    rows = torch.ones(2, 12, dtype=torch.bool, device=DEV)
    rows[1, 5] = rows[0, 6] = rows[1, 8] = False
    assert torch.equal(y[0][rows], base[0][rows]) and torch.isnan(y[0, 1, 5]).all() and not torch.isfinite(y[0, 0, 6]).all()
    pos = torch.arange(12, device=DEV, dtype=torch.int32)
    pos[[5, 6, 8]] = -1  # the same rows belong to nobody: zeros, and nothing in the weights' gradient
    w = torch.ones(64, device=DEV)
    y = R.relation_qk_norm_fwd(z, None, w, None, pos)["q"]
    d = R.relation_qk_norm_bwd(z, None, w, None, z, None, pos)
    assert torch.isfinite(y).all() and not y[0, :, [5, 6, 8]].any()
    assert torch.isfinite(d["dq"]).all() and not d["dq"][0, :, [5, 6, 8]].any() and torch.isfinite(d["dwq"]).all()


def test_empty():
    w = torch.ones(64, device=DEV)
    x = torch.empty(0, 4, 64, device=DEV)
    assert R.relation_qk_norm_fwd(x, x, w, w)["q"].shape == x.shape
    d = R.relation_qk_norm_bwd(x, x, w, w, x, x)
    torch.cuda.synchronize()
    assert not d["dwq"].any() and not d["dwk"].any()


def test_gradients_by_differences_and_through_autograd():
    """Central differences of the forward kernel in fp32 along random directions, step 2^-7: its cubic term and the
    rounding of y leave some 1e-5 of the norms; bar 1e-3. Weights in bf16 get a bf16 gradient."""
    g = torch.Generator(device=DEV).manual_seed(6)
    q, k, dq, dk = (torch.randn(2, h, 30, 48, device=DEV, generator=g) for h in (4, 2, 4, 2))
    wq, wk = (1 + 0.2 * torch.randn(48, device=DEV, generator=g) for _ in range(2))
    kw = dict(rope_dim=32, layout="interleaved", factor=4.0, original_length=512, amplitude=1.1)
    pos = torch.randint(0, 3000, (2, 30), device=DEV, generator=g, dtype=torch.int32)
    leaves = [x.clone().requires_grad_() for x in (q, k, wq, wk)]
    y = R.relation_qk_norm(*leaves, pos, **kw)
    grads = torch.autograd.grad(y, leaves, (dq, dk))

    def f(*x):
        o = R.relation_qk_norm_fwd(*x, pos, **kw)
        return float((o["q"].double() * dq).sum() + (o["k"].double() * dk).sum())
    at, e = [q, k, wq, wk], 2.0 ** -7
    for i in range(4):
        u = torch.randn(at[i].shape, device=DEV, generator=g)
        up, down = ([x + s * e * u if j == i else x for j, x in enumerate(at)] for s in (1, -1))
        num, ana = (f(*up) - f(*down)) / (2 * e), float((grads[i].double() * u).sum())
        assert abs(num - ana) <= 1e-3 * float(grads[i].norm()), (i, num, ana)
    # used by one loss alone, and through views: keys that a loss does not use get zeros
    leaf = q.clone().requires_grad_()
    shared = wq.to(torch.bfloat16).requires_grad_()
    y = R.relation_qk_norm(leaf.to(torch.bfloat16), k.to(torch.bfloat16), shared, shared, pos, **kw)
    y[0].float().sum().backward()
    assert leaf.grad.shape == q.shape and shared.grad.dtype == torch.bfloat16 and torch.isfinite(shared.grad).all()
    y = R.relation_qk_norm(q.requires_grad_(), None, wq.requires_grad_(), None, pos, **kw)
    assert y[1] is None
    y[0].sum().backward()
    with pytest.raises(RuntimeError):
        torch.autograd.grad(torch.autograd.grad(R.relation_qk_norm(q, k, wq, wk, pos)[0].sum(), q, create_graph=True)[0].sum(), q)


def test_repeats_its_bits_on_a_stream_and_in_a_graph():
    g = torch.Generator(device=DEV).manual_seed(7)
    q, k, dq, dk = (torch.randn(2, h, 5000, 64, device=DEV, generator=g).to(torch.bfloat16) for h in (4, 2, 4, 2))
    w = torch.rand(64, device=DEV, generator=g)
    step = lambda: (R.relation_qk_norm_fwd(q, k, w, w), R.relation_qk_norm_bwd(q, k, w, w, dq, dk))
    flat = lambda s: [s[0]["q"], s[0]["k"], s[1]["dq"], s[1]["dk"], s[1]["dwq"], s[1]["dwk"]]
    first = flat(step())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        other = flat(step())
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = flat(step())
    for turn in range(3):
        q.mul_(1.5)
        dk.add_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, flat(step())))


def test_more_than_2_to_the_31_elements():
    """Rows past 32-bit offsets (a view of 4.4 GB with gaps)."""
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 10 GB")
    big = torch.zeros((3, 1 << 30), dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(big, (3, 2, 5, 64), (1 << 30, 64, 1 << 27, 1))
    g = torch.Generator(device=DEV).manual_seed(8)
    x.copy_(torch.randn(x.shape, device=DEV, generator=g))
    a, b = R.relation_qk_norm_fwd(x, None), R.relation_qk_norm_fwd(x.contiguous(), None)
    assert torch.equal(a["q"], b["q"])
    out = {"q": torch.as_strided(torch.zeros_like(big), x.shape, x.stride())}
    assert torch.equal(R.relation_qk_norm_fwd(x.contiguous(), None, out=out)["q"], b["q"])
    del big, x, out
    torch.cuda.empty_cache()


def test_arguments_are_checked():
    x = torch.randn(2, 4, 5, 64, device=DEV)
    w = torch.ones(64, device=DEV)
    for bad in (dict(layout="other"), dict(positions=torch.zeros(4, dtype=torch.int32, device=DEV)), dict(q_weight=w[:32]),
                dict(q_weight=w, norm=False), dict(q_weight=w, k_weight=w.bfloat16()), dict(k=x[..., :32]), dict(k=x.bfloat16()),
                dict(k=x.cpu()), dict(q_weight=w.half())):
        kw = {"q": x, "k": x, **bad}
        with pytest.raises((ValueError, TypeError)):
            R.relation_qk_norm_fwd(kw.pop("q"), kw.pop("k"), **kw)
    for bad in (dict(eps=0.0), dict(eps=math.nan), dict(rope_dim=63), dict(rope_dim=66), dict(rope_base=1.0), dict(factor=0.5),
                dict(original_length=-1), dict(low=3.0, high=3.0), dict(amplitude=math.inf)):
        with pytest.raises(RuntimeError):
            R.relation_qk_norm_fwd(x, x, **bad)
    with pytest.raises(ValueError):
        R.relation_qk_norm_fwd(None, None)
    with pytest.raises(ValueError):
        R.relation_qk_norm_bwd(x, x, None, None, x, None)
    with pytest.raises(TypeError):
        R.relation_qk_norm_fwd(x.half(), None)


def test_outputs_of_the_differentiable_call_are_its_own():
    q = torch.randn((5, 2, 16), device=DEV)
    with pytest.raises(ValueError, match="out"):
        R.relation_qk_norm(q, None, out={"q": torch.empty_like(q)})


def test_rows_of_zeros_and_of_sums_past_32_bits():
    """Zeros stay zeros, forward and back; where the sum of squares passes fp32 the row becomes 0, its neighbours stay."""
    x = torch.randn((4, 2, 64), device=DEV)
    want = R.relation_qk_norm_fwd(x, None)["q"]
    y = x.clone()
    y[1, 0], y[2, 1] = 0.0, 1.0e25
    o = R.relation_qk_norm_fwd(y, None)["q"]
    assert not o[1, 0].any() and not o[2, 1].any()
    keep = torch.ones((4, 2), dtype=torch.bool, device=DEV)
    keep[1, 0] = keep[2, 1] = False
    assert torch.equal(o[keep], want[keep])
    leaf = y.clone().requires_grad_()
    R.relation_qk_norm(leaf, None)[0].sum().backward()
    assert torch.isfinite(leaf.grad).all() and leaf.grad[1, 0].any()  # 1 / sqrt(eps) times the turned ones


@pytest.mark.parametrize("place", ["heads first", "tokens first", "packed"])
def test_outputs_are_worked_on_in_place(place):
    """Scaled and masked in place by the caller: the gradients of the same in 64 bits by hand (bars as above)."""
    g = torch.Generator(device=DEV).manual_seed(5)
    shape = {"heads first": (2, 3, 5, 64), "tokens first": (2, 5, 3, 64), "packed": (10, 3, 64)}[place]
    x = torch.randn(shape, device=DEV, generator=g)
    q = (x.transpose(1, 2) if place == "tokens first" else x).requires_grad_()
    k = q.detach().clone().requires_grad_()
    a, b = R.relation_qk_norm(q, k)
    scale = torch.tensor([0.5, 0.0, 2.0], device=DEV).view((1, 3, 1, 1) if a.dim() == 4 else (1, 3, 1))
    a *= scale
    a[..., :7] = 0.0
    b.mul_(2.0)
    b.masked_fill_(scale == 0, 0.0)
    (a.sum() + (b * b.detach()).sum()).backward()
    da, db = torch.ones_like(a) * scale, b.detach() * 2.0 * (scale != 0)
    da[..., :7] = 0.0
    for leaf, d in ((q, da), (k, db)):
        want = R.relation_qk_norm_bwd(leaf.detach(), None, None, None, d, None)["dq"]
        assert torch.equal(leaf.grad, want)
