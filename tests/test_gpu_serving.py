"""GPU parity of serving from a paged cache (page map, append, decode over pages,
sampling) with the fp64 serving oracle.

Bars. Whole numbers are equal. A row written to the cache or to q_out is an fp32
sum of two products, rounded once: per element 2^-8 of the value in bf16 (2^-23
in fp32), and of what the sum is made of 2^-20 for its fp32 steps and the fp32
sine and cosine. Decode: fp32 arithmetic throughout (relative l2 2e-5: the
exponents reach 40, an fp32 rounding of them 4e-6), one rounding of y (relative
l2 2^-8 in bf16 at most). logprob: 1e-5 absolute and 1e-5 of its exponent."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import serving_oracle as SO
from paper_2608_20172_amd import binding as R
from tests.gpu_helpers import TORCH_DT, log, rel_l2

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    R.load_library()


def _np(t):
    return t.detach().double().cpu().numpy()


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------
# page map
# ---------------------------------------------------------------------------
def _check_map(cached, added, table, free, page, N):
    want = SO.page_map(cached, added, table, free, page, N)
    got = R.relation_page_map(_i32(cached), _i32(added), _i32(table), _i32(free), page, N)
    torch.cuda.synchronize()
    for n, w in want.items():
        assert np.array_equal(got[n].cpu().numpy(), w), n


@pytest.mark.parametrize("B,page,top,add,N,spare", [
    (1, 16, 0, 1, 1, 0), (1, 1, 5, 3, 3, 2), (3, 16, 40, 20, 70, 5), (64, 16, 300, 1, 64, 64), (65, 8, 30, 9, 400, 3),
    (1000, 32, 100, 7, 5000, 100), (1025, 16, 33, 5, 4097, 10000), (4096, 16, 20, 2, 9000, 10000), (7, 128, 500, 3000, 20000, 200),
])
def test_page_map(B, page, top, add, N, spare):
    """Whole and odd batches, more requests than threads, tokens over several workgroups, lists and buffers that end."""
    rng = np.random.default_rng(B * 7 + page)
    cached, added = rng.integers(0, top + 1, B), rng.integers(0, add + 1, B)
    W = (top + add) // page + 1
    table = np.where(np.arange(W)[None] < -(-cached[:, None] // page), rng.permutation(B * W).reshape(B, W), -1)
    log(f"[page_map] B={B} page={page} N={N} free={spare}")
    _check_map(cached, added, table, B * W + rng.permutation(spare), page, N)


def test_page_map_refusals():
    """Negative counts, rows too short, counts near 2^31, a list used up (those that need no page go on)."""
    big = 2 ** 31 - 1
    cached = [-1, 0, 5, big, 16, 17, 3, 0, 40, 0]
    added = [2, -3, 4, big, 16, 1, 0, 33, 1, 1]
    table = np.arange(30).reshape(10, 3)
    for free in (0, 1, 2, 3, 50):
        for N in (0, 5, 30, 100):
            log(f"[page_map] refusals free={free} N={N}")
            _check_map(cached, added, table, np.arange(100, 100 + free), 16, N)


def test_page_map_of_nothing_and_given_outputs():
    empty = torch.empty(0, dtype=torch.int32, device=DEV)
    m = R.relation_page_map(empty, empty, torch.empty((0, 4), dtype=torch.int32, device=DEV), _i32([1]), 16, 3)
    assert m["counts"].tolist() == [0, 0, 0] and m["slots"].tolist() == [-1] * 3 and m["row_start"].tolist() == [0]
    out = {"slots": torch.full((4,), 9, dtype=torch.int64, device=DEV), "lengths": _i32([8, 8])}
    m = R.relation_page_map(_i32([0, 3]), _i32([2, 1]), _i32([[-1], [6]]), _i32([2]), 4, 4, out=out)
    assert m["slots"] is out["slots"] and out["slots"].tolist() == [8, 9, 27, -1] and out["lengths"].tolist() == [2, 4]


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
def _pool(pages, H, page, D, dtype, layout, rng, split=False):
    """k and v pools with some values in them: [P, H, page, D], [P, page, H, D], or both in one allocation."""
    x = torch.from_numpy(rng.standard_normal((2, pages, H, page, D))).to(TORCH_DT[dtype]).to(DEV)
    if layout == "joint":
        both = torch.stack([x[0], x[1]], 1).contiguous()  # [P, 2, H, page, D]
        return both[:, 0], both[:, 1]
    if layout == "nhd":
        return tuple(t.transpose(1, 2).contiguous().transpose(1, 2) for t in x)
    if layout == "wide":  # rows 64 elements apart from each other
        y = torch.zeros((2, pages, H, page, D + 64), dtype=x.dtype, device=DEV)
        y[..., :D] = x
        return y[0][..., :D], y[1][..., :D]
    return x[0].contiguous(), x[1].contiguous()


def _rows_close(name, got, want, parts, dtype):
    got = _np(got)
    bar = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * np.abs(want) + 2.0 ** -20 * parts
    worst = float(np.max(np.abs(got - want) / np.maximum(bar, 1e-30)))
    log(f"  {name}: {worst:.2f} of the bar")
    assert worst <= 1.0, name


@pytest.mark.parametrize("N,H,Hq,D,Dc,page,dtype,layout,pairing,rope", [
    (1, 2, 2, 64, 64, 16, "bf16", "hnd", "A", 1e4), (5, 8, 8, 80, 80, 16, "bf16", "nhd", "B", 1e4),
    (33, 8, 8, 60, 64, 8, "bf16", "hnd", "B", 1e4), (17, 4, 8, 48, 64, 32, "bf16", "joint", "A", 1e4),
    (9, 3, 3, 64, 64, 16, "bf16", "hnd", None, 1e4), (9, 2, 0, 128, 128, 16, "bf16", "nhd", "B", 500.0),
    (12, 1, 7, 32, 40, 1, "bf16", "wide", None, 0.0), (8, 2, 2, 61, 64, 4, "bf16", "hnd", "A", 0.0),
    (4100, 2, 4, 64, 64, 64, "bf16", "nhd", "A", 1e4), (4099, 2, 2, 60, 64, 128, "f32", "hnd", "A", 1e4),
    (6, 2, 2, 80, 80, 16, "f32", "joint", "B", 1e4), (7, 4, 4, 10, 12, 16, "f32", "hnd", "A", 1e4),
    (3, 2, 2, 1, 4, 16, "f32", "nhd", "B", 0.0), (40, 12, 12, 64, 64, 16, "bf16", "nhd", "B", 1e4),
])
def test_append(N, H, Hq, D, Dc, page, dtype, layout, pairing, rope):
    rng = np.random.default_rng(N + D)
    log(f"[append] N={N} H={H} Hq={Hq} D={D} Dc={Dc} page={page} {dtype} {layout} {pairing} rope={rope}")
    pages = N // page + 4
    kc, vc = _pool(pages, H, page, Dc, dtype, layout, rng)
    k0, v0 = _np(kc), _np(vc)
    mk = lambda h: torch.from_numpy(rng.standard_normal((N, h, D))).to(TORCH_DT[dtype]).to(DEV)
    # k and v as halves of a projection, q on its own
    kv = torch.cat([mk(H), mk(H)], 1)
    k, v, q = kv[:, :H], kv[:, H:], mk(Hq) if Hq else None
    slots = rng.permutation(pages * page)[:N]
    positions = np.where(rng.random(N) < 0.3, rng.integers(0, 2 ** 20, N), rng.integers(0, 500, N))
    if N > 4:  # tokens of no request
        slots[1], positions[2], slots[3] = -1, -1, pages * page
    theta = rng.uniform(-math.pi, math.pi, H // 2).astype(np.float32) if pairing else None
    got = R.relation_paged_append(k, v, kc, vc, torch.tensor(slots, device=DEV), _i32(positions), q=q,
                                  theta=None if theta is None else torch.tensor(theta, device=DEV), pairing=pairing,
                                  rope_base=rope)
    torch.cuda.synchronize()
    kw = dict(theta=theta, pairing=pairing, rope_base=rope)
    qn = None if q is None else _np(q)
    wk, wv, wq = SO.append(_np(k), _np(v), k0, v0, slots, positions, q=qn, **kw)
    # what the sums are made of: the pair's two entries, by their larger
    z = np.zeros_like(k0)
    big = max(float(np.abs(_np(kv)).max()), float(np.abs(qn).max()) if qn is not None else 0.0)
    _rows_close("k", kc, wk, np.where(wk == k0, z, big), dtype)
    _rows_close("v", vc, wv, np.where(wv == v0, z, big), dtype)
    if q is not None:
        _rows_close("q", got, wq, np.where(wq == 0, 0.0, big), dtype)
    else:
        assert got is None


def test_append_expanded_rows():
    """Keys of one head for all heads (stride 0) beside values of their own, and the other way round."""
    rng = np.random.default_rng(44)
    N, H, D, page = 5, 4, 64, 16
    one, all_ = (torch.from_numpy(rng.standard_normal((N, h, D))).to(torch.bfloat16).to(DEV) for h in (1, H))
    slots, positions = torch.arange(3, 3 + N, device=DEV), _i32(np.arange(N))
    for k, v in ((one.expand(N, H, D), all_), (all_, one.expand(N, H, D)), (one.expand(N, H, D), one.expand(N, H, D)),
                 (all_[:1].expand(N, H, D), all_)):
        got, want = (_pool(2, H, page, D, "bf16", "hnd", np.random.default_rng(45)) for _ in range(2))
        R.relation_paged_append(k, v, *got, slots, positions)
        R.relation_paged_append(k.contiguous(), v.contiguous(), *want, slots, positions)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("N,H,Hq,D,Dc,page,layout,pairing,rope", [
    (5, 2, 2, 10, 16, 16, "hnd", "A", 1e4), (4100, 2, 1, 14, 16, 8, "nhd", "B", 1e4), (3, 3, 0, 2, 8, 4, "joint", None, 1e4),
    (9, 2, 2, 7, 8, 16, "wide", "A", 0.0), (1, 1, 4, 1, 8, 1, "hnd", None, 0.0),
])
def test_append_narrow_rows(N, H, Hq, D, Dc, page, layout, pairing, rope):
    """bf16 rows, or halves of them with RoPE, under 16 bytes."""
    test_append(N, H, Hq, D, Dc, page, "bf16", layout, pairing, rope)


# ---------------------------------------------------------------------------
# decode
# ---------------------------------------------------------------------------
def _tables(lens, page, rng, extra=2):
    used = -(-np.asarray(lens) // page)
    W = max(1, int(used.max()))
    ids = rng.permutation(int(used.sum()) + extra)
    table = np.full((len(lens), W), -1)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = ids[at:at + n]
        at += n
    return table, int(used.sum()) + extra


def _decode_case(lens, H, G, D, page, dtype, layout="hnd", std=1.0, lam=0.4, seed=0, junk=math.nan, **kw):
    rng = np.random.default_rng(seed + D + page)
    table, pages = _tables(lens, page, rng)
    kc, vc = _pool(pages, H, page, D, dtype, layout, rng)
    kc *= std
    used = np.zeros((pages, page), bool)
    for b, n in enumerate(lens):
        for j in range(n):
            used[table[b, j // page], j % page] = True
    mask = torch.tensor(~used, device=DEV)[:, None, :, None]
    kc.masked_fill_(mask, junk)  # what no request holds
    vc.masked_fill_(mask, junk)
    q = torch.from_numpy(rng.standard_normal((len(lens), H * G, D)) * std).to(TORCH_DT[dtype]).to(DEV)
    lam = float(np.float32(lam))
    r = R.relation_paged_decode(q, kc, vc, _i32(table), _i32(lens), lam, **kw)
    torch.cuda.synchronize()
    Y, M = SO.paged_decode(_np(q), _np(kc), _np(vc), table, lens, lam, **{k: v for k, v in kw.items() if k != "workspace"})
    return r, Y, M, (q, kc, vc, table)


def _decode_close(r, Y, M, dtype):
    ey, em = rel_l2(_np(r["o"]), Y), rel_l2(_np(r["row_stat"]), M)
    bar = 2.0 ** -8 if dtype == "bf16" else 2e-5
    log(f"  y: rel-l2 {ey:.2e} (bar {bar:.1e}); M: {em:.2e} (bar 2e-5)")
    assert ey <= bar and em <= 2e-5


@pytest.mark.parametrize("lens,H,G,D,page,dtype,layout", [
    ([1], 1, 1, 64, 16, "bf16", "hnd"), ([2], 8, 1, 64, 16, "bf16", "nhd"), ([1, 2, 3, 16, 17], 2, 2, 32, 16, "bf16", "hnd"),
    ([256, 257, 258, 511, 512, 513], 2, 1, 64, 16, "bf16", "hnd"), ([700, 5, 1], 3, 4, 80, 8, "bf16", "nhd"),
    ([1025, 33], 2, 3, 96, 32, "bf16", "joint"), ([300], 1, 8, 128, 64, "bf16", "hnd"), ([290], 2, 5, 48, 1, "bf16", "wide"),
    ([2047, 41, 1000], 4, 1, 80, 16, "f32", "hnd"), ([257, 100], 2, 4, 128, 128, "f32", "nhd"), ([77], 1, 3, 4, 16, "f32", "hnd"),
    ([40, 1, 9], 2, 7, 8, 4, "bf16", "hnd"), ([5000], 2, 1, 64, 512, "bf16", "nhd"), ([4097, 17], 1, 6, 128, 16, "bf16", "joint"),
    ([3000, 2999, 1], 2, 2, 128, 1024, "f32", "hnd"), ([600] * 40 + [3] * 30, 3, 1, 64, 16, "bf16", "hnd"),
    ([1300] * 20, 2, 16, 64, 16, "bf16", "hnd"), ([900] * 9, 1, 9, 112, 16, "bf16", "nhd"), ([500, 20], 2, 12, 120, 16, "f32", "hnd"),
])
def test_paged_decode(lens, H, G, D, page, dtype, layout):
    log(f"[paged_decode] lens={lens[:6]} H={H} G={G} D={D} page={page} {dtype} {layout}")
    r, Y, M, (_, _, vc, table) = _decode_case(lens, H, G, D, page, dtype, layout)
    _decode_close(r, Y, M, dtype)
    for b, n in enumerate(lens):  # one token: y is its own value exactly
        if n == 1:
            assert torch.equal(r["o"][b], vc[table[b, 0], :, 0].repeat_interleave(G, 0))


@pytest.mark.parametrize("D,Dc,dtype", [(60, 64, "bf16"), (48, 64, "bf16"), (80, 96, "bf16"), (60, 64, "f32"), (10, 12, "f32")])
def test_padded_heads_decode_as_the_whole_sequence(D, Dc, dtype):
    """Rows of a width that the cache pads, appended and decoded with the true width given: the last row of
    relation_layer_fwd on the same heads, whose scale is 1/sqrt of the true width."""
    rng = np.random.default_rng(51 + D)
    T, H, page = 130, 4, 16
    q, k, v = (torch.from_numpy(rng.standard_normal((T, H, D)) * 2.0).to(TORCH_DT[dtype]).to(DEV) for _ in range(3))
    theta = torch.from_numpy(rng.uniform(-1, 1, H // 2)).float().to(DEV)
    pages = -(-T // page)
    kc, vc = (torch.zeros((pages, H, page, Dc), dtype=TORCH_DT[dtype], device=DEV) for _ in range(2))
    table = _i32(rng.permutation(pages)[None])
    m = R.relation_page_map(_i32([0]), _i32([T]), torch.zeros_like(table), table[0], page, T)
    qr = R.relation_paged_append(k, v, kc, vc, m["slots"], m["positions"], q=q, theta=theta, pairing="A")
    y = R.relation_paged_decode(qr[-1:], kc, vc, m["table"], m["lengths"], 0.5, head_dim=D)
    torch.cuda.synchronize()
    Y, M = SO.paged_decode(_np(qr[-1:]), _np(kc), _np(vc), _np(m["table"]).astype(int), [T], 0.5, scale=D ** -0.5)
    _decode_close(y, Y, M, dtype)
    w = R.relation_layer_fwd(*(t.transpose(0, 1)[None] for t in (q, k, v)), 0.5, theta, pairing="A")["o"][0, :, -1]
    # bf16: both paths round q, k, v and y once each, and the whole sequence its weights: a few times 2^-8. fp32: the
    # whole sequence's bar is 1e-4 of entries of some 0.3 and more, the decode step's 2e-5
    err, bar = rel_l2(_np(y["o"][0, :, :D]), _np(w)), 2.0 ** -8 * 4 if dtype == "bf16" else 4e-4
    log(f"[padded heads] D={D} Dc={Dc} {dtype}: {err:.2e} of the whole sequence's row (bar {bar:.1e})")
    assert err <= bar and not y["o"][:, :, D:].any()


def test_paged_decode_head_dim_is_checked():
    kc, vc = _pool(2, 2, 16, 64, "bf16", "hnd", np.random.default_rng(53))
    q, table, lens = kc[:1, :, 0].contiguous(), _i32([[0, 1]]), _i32([5])
    for bad in (dict(head_dim=0), dict(head_dim=65), dict(head_dim=60, scale=0.1)):
        with pytest.raises(ValueError, match="head_dim"):
            R.relation_paged_decode(q, kc, vc, table, lens, 0.5, **bad)
    a, b = (R.relation_paged_decode(q, kc, vc, table, lens, 0.5, **kw) for kw in (dict(head_dim=64), dict()))
    assert torch.equal(a["o"], b["o"]) and torch.equal(a["row_stat"], b["row_stat"])


@pytest.mark.parametrize("B,H,G,D,dtype", [(64, 3, 1, 48, "bf16"), (67, 2, 17, 80, "bf16"), (71, 3, 1, 40, "f32"),
                                           (65, 2, 6, 20, "f32")])
def test_paged_decode_heads_that_share_lines(B, H, G, D, dtype):
    """Heads side by side in rows that are no multiple of 128 bytes, with over 64 slices and requests: groups of
    workgroups are placed, 64 of them to 71 (full turns of eight and broken ones), one slice a row and several."""
    for top in (200, 700):
        lens = [1 + (37 * b) % top for b in range(B)]
        log(f"[paged_decode] placed B={B} H={H} G={G} D={D} {dtype} up to {top}")
        r, Y, M, _ = _decode_case(lens, H, G, D, 16, dtype, "nhd")
        _decode_close(r, Y, M, dtype)


@pytest.mark.parametrize("B,H,G,D,top,page,dtype", [(300, 8, 1, 32, 1500, 16, "bf16"), (40, 8, 2, 64, 5000, 1, "bf16"),
                                                    (150, 8, 1, 32, 1400, 32, "f32"), (24, 16, 1, 128, 3300, 256, "bf16")])
def test_paged_decode_many_rows(B, H, G, D, top, page, dtype):
    """So many rows that a slice is long: one of 4096 keys a row, several of 512 to 2048, offsets of 2048 pages of one
    token."""
    lens = [1 + (top * (b + 1) // B * 7919) % top for b in range(B)]
    log(f"[paged_decode] many rows B={B} H={H} G={G} D={D} up to {max(lens)} page={page} {dtype}")
    r, Y, M, _ = _decode_case(lens, H, G, D, page, dtype, "hnd")
    _decode_close(r, Y, M, dtype)


@pytest.mark.parametrize("D,B,H", [(128, 50, 16), (32, 80, 10)])
def test_paged_decode_long_slices_of_one_token_pages(D, B, H):
    """Slices of 4096 pages of one token: the largest tables in LDS, beside the widest rows' tiles. The requests share
    pages, and few of them are as long as the bound."""
    rng = np.random.default_rng(62)
    kc, vc = _pool(700, H, 1, D, "bf16", "hnd", rng)
    W = 6000
    table = rng.integers(0, 700, (B, W))
    lens = np.where(np.arange(B) < 2, [W - b for b in range(B)], 1 + np.arange(B) * 7)
    q = torch.from_numpy(rng.standard_normal((B, H, D))).to(torch.bfloat16).to(DEV)
    log(f"[paged_decode] one-token pages D={D} B={B} H={H}")
    r = R.relation_paged_decode(q, kc, vc, _i32(table), _i32(lens), 0.5)
    torch.cuda.synchronize()
    some = [0, 1, 2, B - 1]
    Y, M = SO.paged_decode(_np(q[some]), _np(kc), _np(vc), table[some], lens[some], 0.5)
    _decode_close({n: t[some] for n, t in r.items()}, Y, M, "bf16")


def test_paged_decode_long():
    """One request of 40000 tokens, 4 heads of width 128: many slices, 157 of them of 256 keys."""
    r, Y, M, _ = _decode_case([40000, 3], 4, 1, 128, 64, "bf16", "nhd")
    _decode_close(r, Y, M, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 6])
def test_paged_decode_sharp(dtype, G):
    """Evidence of tens of units: the running maximum moves; and scale, tau_s, lambda and max_length given."""
    r, Y, M, _ = _decode_case([777, 130, 64], 2, G, 64, 16, dtype, std=3.0, lam=-0.7, max_length=777)
    _decode_close(r, Y, M, dtype)
    r, Y, M, _ = _decode_case([600, 130, 1], 2, G, 64, 16, dtype, std=1.5, lam=2.0, scale=0.3, tau_s=0.5, max_length=640)
    _decode_close(r, Y, M, dtype)


@pytest.mark.parametrize("G", [1, 4, 8])
def test_paged_decode_bad_lengths_and_pages(G):
    """Lengths outside 1 .. the bound and pages outside the pool give NaN rows of that request alone, and pages past
    a request's length are never looked at."""
    rng = np.random.default_rng(9)
    lens = [30, 30, 30, 30, 30, 30, 600, 600]
    table, pages = _tables(lens, 16, rng)
    kc, vc = _pool(pages, 2, 16, 64, "bf16", "hnd", rng)
    q = torch.from_numpy(rng.standard_normal((8, 2 * G, 64))).to(torch.bfloat16).to(DEV)
    given = np.array([0, -5, 30, 10 ** 9, 30, 30, 601, 600])
    table[4, 0], table[5, 1], table[7, 20] = pages, -1, 2 ** 31 - 1
    table[2, 2:] = -7
    r = R.relation_paged_decode(q, kc, vc, _i32(table), _i32(given), 0.2, max_length=600)
    torch.cuda.synchronize()
    Y, M = SO.paged_decode(_np(q), _np(kc), _np(vc), table, given, 0.2, max_length=600)
    assert np.array_equal(np.isnan(_np(r["o"])), np.isnan(Y)) and np.array_equal(np.isnan(_np(r["row_stat"])), np.isnan(M))
    assert not np.isnan(Y[2]).any() and np.isnan(Y[[0, 1, 3, 4, 5, 6, 7]]).all()
    assert rel_l2(_np(r["o"])[2], Y[2]) <= 2.0 ** -8


@pytest.mark.parametrize("G,D", [(1, 64), (8, 128)])
def test_paged_decode_nan_in_the_history_stays_in_its_rows(G, D):
    r, _, _, (q, kc, vc, table) = _decode_case([400, 400], 2, G, D, 16, "bf16")
    vc[table[0, 3], 1, 2] = math.nan
    n = R.relation_paged_decode(q, kc, vc, _i32(table), _i32([400, 400]), 0.4)
    torch.cuda.synchronize()
    assert torch.isnan(n["o"][0, G:]).all() and torch.equal(n["o"][0, :G], r["o"][0, :G]) and torch.equal(n["o"][1], r["o"][1])
    assert torch.equal(n["row_stat"], r["row_stat"])  # no value enters M
    kc[table[1, 0], 0, 0] = math.nan
    n = R.relation_paged_decode(q, kc, vc, _i32(table), _i32([400, 400]), 0.4)
    torch.cuda.synchronize()
    assert torch.isnan(n["o"][1, :G]).all() and torch.isnan(n["row_stat"][1, :G]).all()
    assert torch.equal(n["row_stat"][1, G:], r["row_stat"][1, G:])


def test_paged_decode_is_decode_on_a_contiguous_cache():
    """The same rows as relation_decode against the same cache laid out contiguously, and the same bits twice."""
    rng = np.random.default_rng(11)
    lens, H, D, page, Tmax = [300, 1, 64], 4, 64, 16, 304
    k, v = (torch.from_numpy(rng.standard_normal((3, H, Tmax, D))).to(torch.bfloat16).to(DEV) for _ in range(2))
    q = torch.from_numpy(rng.standard_normal((3, H, D))).to(torch.bfloat16).to(DEV)
    perm = torch.tensor(rng.permutation(3 * Tmax // page), device=DEV)
    paged = [torch.empty((len(perm), H, page, D), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for p, x in zip(paged, (k, v)):
        p[perm] = x.view(3, H, Tmax // page, page, D).transpose(1, 2).reshape(-1, H, page, D)
    a = R.relation_paged_decode(q, *paged, perm.view(3, -1), _i32(lens), 0.5)
    b = R.relation_paged_decode(q, *paged, perm.view(3, -1), _i32(lens), 0.5)
    c = R.relation_decode(q, k, v, _i32(lens), 0.5)
    torch.cuda.synchronize()
    assert torch.equal(a["o"], b["o"]) and torch.equal(a["row_stat"], b["row_stat"])
    assert rel_l2(_np(a["o"]), _np(c["o"])) <= 2.0 ** -8 and rel_l2(_np(a["row_stat"]), _np(c["row_stat"])) <= 2e-5


def test_paged_offsets_past_32_bits():
    """A pool of over 2^32 elements (9 GB in bf16): rows written to its last pages and read from them."""
    pages, H, page, D = 8200, 16, 256, 128  # 2^32 + 2^23 elements
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 20 GB")
    kc, vc = (torch.zeros((pages, H, page, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rng = np.random.default_rng(12)
    n = 300
    table = np.array([[8199, 8197]])
    slots = np.array([table[0, j // page] * page + j % page for j in range(n)])
    k, v = (torch.from_numpy(rng.standard_normal((n, H, D))).to(torch.bfloat16).to(DEV) for _ in range(2))
    R.relation_paged_append(k, v, kc, vc, torch.tensor(slots, device=DEV), _i32(np.arange(n)), rope_base=None)
    q = torch.from_numpy(rng.standard_normal((1, H, D))).to(torch.bfloat16).to(DEV)
    r = R.relation_paged_decode(q, kc, vc, _i32(table), _i32([n]), 0.5)
    torch.cuda.synchronize()
    assert torch.equal(kc[8199, :, 7], k[7]) and torch.equal(vc[8197, :, 43], v[299]) and not kc[:8000].any()
    small = [x[[8197, 8199]].contiguous() for x in (kc, vc)]
    del kc, vc
    Y, M = SO.paged_decode(_np(q), _np(small[0]), _np(small[1]), [[1, 0]], [n], 0.5)
    _decode_close(r, Y, M, "bf16")
    torch.cuda.empty_cache()


def test_whole_numbers_past_32_bits_keep_their_meaning():
    """int64 lengths, pages, counts and filters of 2^32 and more are out of range as they stand, not the small number
    that their low half makes."""
    i64 = lambda x: torch.tensor(x, dtype=torch.int64, device=DEV)
    far = 1 << 32
    m = R.relation_page_map(i64([far + 1, 0, 3]), i64([1, far + 2, -far + 1]), _i32([[5, 6], [-1, -1], [7, -1]]),
                            i64([1, 2]), 4, 8)
    assert m["counts"].tolist() == [0, 0, 3] and m["lengths"].tolist() == [0, 0, 0]
    assert m["table"].tolist() == [[5, 6], [-1, -1], [7, -1]] and m["row_start"].tolist() == [0, 1, 8, 8]
    m = R.relation_page_map(i64([0]), i64([1]), _i32([[-1]]), i64([far + 9]), 4, 1)
    assert not 0 <= int(m["slots"][0]) // 4 < 1 << 28
    rng = np.random.default_rng(41)
    kc, vc = _pool(8, 2, 16, 64, "bf16", "hnd", rng)
    q = torch.from_numpy(rng.standard_normal((3, 2, 64))).to(torch.bfloat16).to(DEV)
    y = R.relation_paged_decode(q, kc, vc, i64([[1, 2], [3, far + 4], [5, 6]]), i64([20, 20, far + 20]), 0.5)
    assert not torch.isnan(y["o"][0]).any() and torch.isnan(y["o"][1:]).all() and torch.isnan(y["row_stat"][1:]).all()
    k = torch.from_numpy(rng.standard_normal((3, 2, 64))).to(torch.bfloat16).to(DEV)
    before = kc.clone()
    R.relation_paged_append(k, k, kc, vc, i64([0, 17, 35]), i64([far + 1, 4, -far + 1]), rope_base=None)
    assert torch.equal(kc[1, :, 1], k[1])
    kc[1, :, 1] = before[1, :, 1]
    assert torch.equal(kc, before)
    x = torch.zeros((2, 100), device=DEV)
    x[:, 50] = 1.0
    noise = torch.ones_like(x)
    noise[:, 7] = 1e-6
    t = R.relation_sample(x, noise, top_k=i64([far + 1, 1]))["tokens"]
    assert t.tolist() == [7, 50]


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
CLEAR = 1e-5  # what is nearer than this to going the other way is fp32's to choose


def _sure_sample(x, noise, T, k, p, mp):
    """The oracle's sample, and whether its token stays the same with the filters' bounds moved by CLEAR either way
    and the race's second moved up by it."""
    w = [SO.sample(x, noise, T, k, p * s if p < 1 else p, mp * s) for s in (1.0, 1.0 + CLEAR, 1.0 - CLEAR)]
    return w[0], all(y["token"] == w[0]["token"] and not 0 < y["lead"] < CLEAR for y in w)


def _check_sample(x, noise, T=1.0, k=0, p=1.0, mp=0.0, clear=0.9):
    """x, noise: [B, V] device tensors; parameters: numbers or lists of B. At least `clear` of the rows are sure."""
    B = x.shape[0]
    col = lambda v: list(v) if isinstance(v, (list, tuple, np.ndarray)) else [v] * B
    T, k, p, mp = col(T), col(k), col(p), col(mp)
    f = lambda v, t: torch.tensor(v, dtype=t, device=DEV)
    r = R.relation_sample(x, noise, temperature=f(T, torch.float32), top_k=f(k, torch.int32), top_p=f(p, torch.float32),
                          min_p=f(mp, torch.float32))
    torch.cuda.synchronize()
    tokens, lp = r["tokens"].cpu().numpy(), _np(r["logprob"])
    xn, nn = _np(x), _np(noise)
    sure = 0
    for b in range(B):
        w, ok = _sure_sample(xn[b], nn[b], float(np.float32(T[b])), k[b], float(np.float32(p[b])), float(np.float32(mp[b])))
        if not ok:
            log(f"  row {b}: nearer than {CLEAR} to another token")
            continue
        sure += 1
        assert tokens[b] == w["token"], (b, T[b], k[b], p[b], mp[b], tokens[b], w["token"], w["lead"], len(w["kept"]))
        if math.isnan(w["logprob"]):
            assert math.isnan(lp[b])
        else:
            assert abs(lp[b] - w["logprob"]) <= 1e-5 * (1 + abs(w["logprob"])), (b, lp[b], w["logprob"])
    assert sure >= clear * B, f"{sure} of {B} rows are sure"


def _logits(B, V, dtype, rng, slope=1.2, ranked=False):
    rank = np.arange(V)[None] if ranked else rng.random((B, V)) * V
    x = -slope * np.log1p(rank) + 0.3 * rng.standard_normal((B, V))
    return torch.from_numpy(x).to(TORCH_DT[dtype]).to(DEV)


def _noise(B, V, rng):
    return torch.from_numpy(rng.exponential(size=(B, V))).float().to(DEV)


@pytest.mark.parametrize("B,V,dtype,ranked", [
    (1, 1, "f32", False), (2, 2, "bf16", False), (3, 7, "f32", False), (5, 63, "bf16", True), (4, 65, "f32", True),
    (3, 1000, "bf16", False), (2, 1023, "f32", True), (2, 8192, "bf16", False), (2, 8193, "f32", False),
    (3, 32000, "f32", True), (2, 50257, "bf16", True), (1, 131072, "f32", False), (1, 200003, "bf16", False),
])
def test_sample_sizes(B, V, dtype, ranked):
    rng = np.random.default_rng(V)
    log(f"[sample] B={B} V={V} {dtype} ranked={ranked}")
    x, r = _logits(B, V, dtype, rng, ranked=ranked), _noise(B, V, rng)
    _check_sample(x, r)
    _check_sample(x, r, T=0.0, k=5, p=0.3)
    _check_sample(x, r, T=0.7, k=50, p=0.9, mp=0.01)
    _check_sample(x, r, T=1.3, p=0.97)


def test_sample_parameters():
    """Every row its own filters, from none to those that leave one token, over 200 rows."""
    B, V = 200, 4099
    rng = np.random.default_rng(21)
    for dtype in ("f32", "bf16"):
        x, r = _logits(B, V, dtype, rng), _noise(B, V, rng)
        T = rng.choice([0.0, 0.05, 0.6, 1.0, 1.0, 3.0], B)
        k = rng.choice([0, 0, -1, 1, 2, 40, 1000, 4098, 4099, 10 ** 6], B)
        p = rng.choice([1.0, 1.0, 1.5, 0.0, -1.0, 0.3, 0.9, 0.999], B)
        mp = rng.choice([0.0, 0.0, -1.0, 0.001, 0.1, 1.0, 2.0], B)
        log(f"[sample] parameters {dtype}")
        _check_sample(x, r, T, k.tolist(), p, mp)


@pytest.mark.parametrize("B,V,dtype,ranked", [(40, 60001, "f32", False), (33, 70007, "bf16", True), (2, 600011, "bf16", False),
                                              (1, 2097152, "f32", False)])
def test_sample_whole_chunks(B, V, dtype, ranked):
    """Rows in chunks of 8192: many of them, or very long ones; every row its own filters, flat nuclei among them."""
    rng = np.random.default_rng(26 + V)
    x, r = _logits(B, V, dtype, rng, slope=1.1, ranked=ranked), _noise(B, V, rng)
    log(f"[sample] whole chunks B={B} V={V} {dtype} ranked={ranked}")
    T = rng.choice([0.0, 0.6, 1.0, 1.3], B)
    k = rng.choice([0, 0, 1, 40, 1000, 20000], B)
    p = rng.choice([1.0, 0.3, 0.9, 0.97], B)
    mp = rng.choice([0.0, 0.0, 0.001, 0.1], B)
    _check_sample(x, r, T, k.tolist(), p, mp)
    _check_sample(x, r, 1.3, 0, 0.9, 0.0)
    _check_sample(x, r)


def test_sample_is_the_same_every_time():
    """The same bits in every run, whatever the order in which workgroups and waves arrive."""
    rng = np.random.default_rng(27)
    for B, V, dtype in ((3, 5000, "bf16"), (5, 50257, "f32"), (64, 40000, "bf16")):
        x, r = _logits(B, V, dtype, rng), _noise(B, V, rng)
        par = dict(temperature=1.2, top_k=None, top_p=0.93, min_p=None)
        a = R.relation_sample(x, r, **par)
        for _ in range(4):
            b = R.relation_sample(x, r, **par)
            assert torch.equal(a["tokens"], b["tokens"]) and torch.equal(a["logprob"], b["logprob"])


@pytest.mark.parametrize("V", [600, 20000, 131072])
def test_sample_flat_and_tied_rows(V):
    """Rows without a peak: all equal, two values, a slow slope; nuclei of nearly all tokens, and ties at every edge."""
    rng = np.random.default_rng(22)
    flat = np.zeros((6, V))
    flat[1] = rng.integers(0, 2, V)
    flat[2] = -np.arange(V) * 1e-5
    flat[3] = rng.integers(-3, 1, V)
    flat[4] = -np.arange(V)[::-1] * 1e-5
    flat[5] = np.sort(rng.standard_normal(V))
    r = _noise(6, V, rng)
    for dtype in ("f32", "bf16"):
        x = torch.from_numpy(flat).to(TORCH_DT[dtype]).to(DEV)
        log(f"[sample] flat V={V} {dtype}")
        for kw in (dict(), dict(p=0.5), dict(k=V // 3), dict(k=7), dict(k=V // 2, p=0.8, mp=0.4)):
            _check_sample(x, r, **kw)


@pytest.mark.parametrize("V", [500, 40000])
def test_sample_masks_and_infinities(V):
    low = float(torch.finfo(torch.float32).min)
    rng = np.random.default_rng(23)
    x = rng.standard_normal((12, V)) * 2
    x[0] = -np.inf
    x[1] = np.nan
    x[2] = low
    x[3, : V // 2] = -np.inf
    x[4, ::2] = low
    x[5, 3] = np.nan
    x[6] = -np.inf
    x[6, V - 1] = -4.0
    x[7, 17] = np.inf
    x[8, [5, 9]] = np.inf
    x[9] = np.nan
    x[9, 100] = 1.0
    x[10, 1:] = low
    x[11] = 3.0e38
    r = _noise(12, V, rng)
    r[:, 0] = 0.0
    r[5, 8] = -1.0
    for dtype in ("f32", "bf16"):
        y = torch.from_numpy(x).to(torch.float32).to(TORCH_DT[dtype]).to(DEV)
        log(f"[sample] masks V={V} {dtype}")
        for kw in (dict(), dict(T=0.0), dict(k=20, p=0.9), dict(p=0.95, mp=0.01), dict(T=1e-30), dict(T=math.inf)):
            _check_sample(y, r, **kw)
    y = torch.zeros((5, V), device=DEV)
    bad = R.relation_sample(y, torch.ones_like(y), temperature=torch.tensor([-1.0, math.nan, 1, 1, 1], device=DEV),
                            top_p=torch.tensor([1, 1, math.nan, 1, 1.0], device=DEV),
                            min_p=torch.tensor([0, 0, 0, math.nan, 0.0], device=DEV))
    assert bad["tokens"].tolist() == [-1] * 4 + [0] and torch.isnan(bad["logprob"][:4]).all()


@pytest.mark.parametrize("V", [500, 40000])
def test_sample_subnormal_temperatures(V):
    """Temperatures under 2^-126: the largest logits share the weight, whatever their size, and logits that differ by
    as little as the temperature keep their weights."""
    rng = np.random.default_rng(28 + V)
    tiny = float(np.float32(1e-40))
    x = rng.standard_normal((9, V))
    x[1] = 0.0
    x[2, [7, 11, V - 1]] = 9.0
    x[3] = -np.arange(V) * tiny           # weights exp(-0), exp(-1), exp(-2), ...
    x[4] = -np.arange(V)[::-1] * tiny
    x[5] = np.where(rng.random(V) < 0.5, 3.0e38, 2.9e38)
    x[6, [3, V // 2]] = np.inf
    x[7] = -np.inf
    x[7, [5, 6]] = -1.0e38
    x[8] = 1.0 + 2.0 ** -7 * rng.integers(0, 2, V)
    r = _noise(9, V, rng)
    for dtype in ("f32", "bf16"):
        y = torch.from_numpy(x).to(torch.float32).to(TORCH_DT[dtype]).to(DEV)
        log(f"[sample] subnormal T V={V} {dtype}")
        for kw in (dict(T=1e-40), dict(T=4.2e-39, p=0.9), dict(T=1.5e-45, k=20, p=0.95), dict(T=1e-39, mp=0.1),
                   dict(T=1e-38)):
            _check_sample(y, r, **kw)


def test_sample_several_tokens_from_one_row():
    """Expanded logits (row stride 0) are read where they are, as their copies would be; expanded noise as well."""
    rng = np.random.default_rng(29)
    for V, dtype in ((1, "f32"), (300, "f32"), (20001, "bf16")):
        x, r = _logits(1, V, dtype, rng), _noise(6, V, rng)
        par = dict(temperature=0.9, top_k=40, top_p=0.95)
        a, b = (R.relation_sample(y, r, **par) for y in (x.expand(6, V), x.expand(6, V).contiguous()))
        assert torch.equal(a["tokens"], b["tokens"]) and torch.equal(a["logprob"], b["logprob"])
        _check_sample(x.expand(6, V), r, T=0.9, k=40, p=0.95)
        c = R.relation_sample(x.expand(6, V), r[:1].expand(6, V), **par)["tokens"]
        assert c.tolist() == [int(c[0])] * 6


@pytest.mark.parametrize("V,dtype", [(8192, "f32"), (16384, "bf16"), (9000, "f32"), (131072, "f32"), (131072, "bf16"), (1 << 20, "f32")])
def test_sample_random_numbers_in_the_order_of_the_logits(V, dtype):
    """Random numbers that fall along the order of the logits: the race's winner is always the last token left, and the
    kept tokens are found all the same, in a time that the number of tokens does not multiply."""
    # neighbours in the race are 3.6e-5 apart at least, and a level of 1000 gains more by them than it loses by its logit
    step = np.arange(V) // 1000
    x = np.zeros((8, V))
    x[2:5] = -(2.0 ** -6) * step
    x[5] = -(2.0 ** -6) * step[::-1]
    x[6] = -np.arange(V) * 2.0 ** -18
    x[7, V // 2:] = np.inf
    w = np.exp(-(2.0 ** -6) * step)
    before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
    at = 5432                                                          # kept by top-p: tokens 0 .. at
    p = (before[at] + 0.5 * w[at]) / w.sum()
    k = [V // 3, V - 1, 0, 0, 3500, 2999, V // 3, V // 5]
    top_p = [1.0, 1.0, p, 1.0, 0.9999, 1.0, 1.0, 1.0]
    min_p = [0.0, 0.0, 0.0, math.exp(-(2.0 ** -6) * 4.5), 0.0, 0.0, 0.0, 0.0]
    y = torch.from_numpy(x).to(torch.float32).to(TORCH_DT[dtype]).to(DEV)
    r = (3.0 * torch.exp(-4e-5 * torch.arange(V, dtype=torch.float64))).float().to(DEV).expand(8, V).contiguous()
    r[5] = r[5].flip(0)
    log(f"[sample] numbers in the logits' order V={V} {dtype}")
    _check_sample(y, r, 1.0, k, top_p, min_p)
    if V < 1 << 20:
        _check_sample(y, r, 1.0, 0, 0.0, 0.0)
        _check_sample(y, r, 1.0, 0, 1.0, 2.0)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    R.relation_sample(y, r, top_k=_i32(k))
    end.record()
    torch.cuda.synchronize()
    log(f"  {start.elapsed_time(end):.2f} ms")
    assert start.elapsed_time(end) < 5.0 + V / 2000  # a round for each token left out would be over 0.02 V


def test_sample_strides_and_alignment():
    """Rows off 16-byte boundaries, rows apart from each other, rows read backwards from a transpose, no parameters."""
    rng = np.random.default_rng(24)
    big = _logits(5, 3001, "bf16", rng)
    noise = _noise(5, 3500, rng)
    for a, n in ((1, 3000), (3, 2500), (7, 1001)):
        _check_sample(big[:, a:a + n], noise[:, a:a + n], k=30, p=0.9)
        _check_sample(big.float()[:, a:a + n], noise[:, a + 1:a + 1 + n], p=0.99)
    _check_sample(big.t().contiguous().t(), noise[:, :3001], k=30)
    r = R.relation_sample(big, noise[:, :3001].contiguous())
    s = R.relation_sample(big, noise[:, :3001], temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
    assert torch.equal(r["tokens"], s["tokens"]) and torch.equal(r["logprob"], s["logprob"])


def test_sample_frequencies():
    """Tokens of one row drawn 40000 times come as often as the kept weights say."""
    V, n = 300, 40000
    rng = np.random.default_rng(25)
    x = _logits(1, V, "f32", rng).expand(n, V)
    g = torch.Generator(device=DEV).manual_seed(5)
    noise = torch.empty(n, V, device=DEV).exponential_(generator=g)
    t = R.relation_sample(x.contiguous(), noise, temperature=0.8, top_k=40, top_p=0.9)["tokens"].cpu().numpy()
    xs = _np(x[0])
    kept = SO.sample(xs, np.ones(V), float(np.float32(0.8)), 40, float(np.float32(0.9)))["kept"]
    w = np.exp(xs[kept] / 0.8)
    w /= w.sum()
    hits = np.bincount(t, minlength=V)
    assert hits.sum() == hits[kept].sum()
    assert np.all(np.abs(hits[kept] / n - w) < 5 * np.sqrt(w * (1 - w) / n))


def test_outputs_and_workspaces_of_the_caller():
    """out= and workspace= of append, decode and sample: the same values, in the caller's tensors; what does not fit is
    refused."""
    rng = np.random.default_rng(61)
    B, H, D, page, W = 3, 2, 64, 16, 100
    kc, vc = _pool(B * W, H, page, D, "bf16", "hnd", rng)
    table = torch.arange(B * W, dtype=torch.int32, device=DEV).view(B, W)
    lens = _i32([1600, 1, 900])
    k = torch.from_numpy(rng.standard_normal((B, H, D))).to(torch.bfloat16).to(DEV)
    slots = torch.tensor([1599, 1600, 3200 + 899], device=DEV)
    want = R.relation_paged_append(k, k, kc, vc, slots, lens - 1, q=k)
    out = {"q": torch.full_like(want, 9.0)}
    assert R.relation_paged_append(k, k, kc, vc, slots, lens - 1, q=k, out=out) is out["q"] and torch.equal(out["q"], want)
    y = R.relation_paged_decode(want, kc, vc, table, lens, 0.5)
    c, d = R.make_pages(kc, vc), R.RelPagedQuery(B, H, W, 0, 2.0, 0.0)
    need = R.load_library().relation_paged_decode_workspace_bytes(R.ctypes.byref(c), R.ctypes.byref(d))
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    out = {"o": torch.full_like(want, 9.0), "row_stat": torch.full((B, H), 9.0, device=DEV)}
    got = R.relation_paged_decode(want, kc, vc, table, lens, 0.5, workspace=ws, out=out)
    assert got["o"] is out["o"] and got["row_stat"] is out["row_stat"]
    assert torch.equal(out["o"], y["o"]) and torch.equal(out["row_stat"], y["row_stat"])
    x, r = _logits(B, 20000, "f32", rng), _noise(B, 20000, rng)
    s = R.relation_sample(x, r, top_p=0.9)
    need = R.load_library().relation_sample_workspace_bytes(R.ctypes.byref(R.RelSample(B, 20000, R.REL_F32, 20000, 20000)))
    assert need > 0
    sws = torch.empty(need, dtype=torch.uint8, device=DEV)
    out = {"tokens": torch.full((B,), 9, device=DEV), "logprob": torch.full((B,), 9.0, device=DEV)}
    got = R.relation_sample(x, r, top_p=0.9, workspace=sws, out=out)
    assert got["tokens"] is out["tokens"] and got["logprob"] is out["logprob"]
    assert torch.equal(out["tokens"], s["tokens"]) and torch.equal(out["logprob"], s["logprob"])
    small = torch.empty(16, dtype=torch.uint8, device=DEV)  # one that is too small is not used
    assert torch.equal(R.relation_paged_decode(want, kc, vc, table, lens, 0.5, workspace=small)["o"], y["o"])
    assert torch.equal(R.relation_sample(x, r, top_p=0.9, workspace=small)["tokens"], s["tokens"])
    with pytest.raises(ValueError, match="contiguous"):
        R.relation_paged_decode(want, kc, vc, table, lens, 0.5, out={"o": y["o"][:2]})
    with pytest.raises(ValueError, match="contiguous"):
        R.relation_sample(x, r, top_p=0.9, out={"tokens": s["tokens"].int()})
    with pytest.raises(ValueError, match="contiguous"):
        R.relation_paged_append(k, k, kc, vc, slots, lens - 1, q=k, out={"q": want.float()})


# ---------------------------------------------------------------------------
# streams and graphs
# ---------------------------------------------------------------------------
def test_serving_on_a_stream_and_in_a_graph():
    """The whole step on a stream of its own, recorded once and replayed with other inputs, against eager calls."""
    rng = np.random.default_rng(31)
    B, H, D, page, V, W = 6, 4, 64, 16, 5000, 40
    kc, vc = _pool(B * W, H, page, D, "bf16", "hnd", rng)
    table = torch.arange(B * W, dtype=torch.int32, device=DEV).view(B, W).contiguous()
    free = torch.empty(0, dtype=torch.int32, device=DEV)
    cached = _i32([3, 100, 200, 17, 599, 16 * 33])
    # pages of every request are in the table: cached is rounded so that a step needs none
    one = _i32([1] * B)
    q, k, v = (torch.from_numpy(rng.standard_normal((B, H, D))).to(torch.bfloat16).to(DEV) for _ in range(3))
    logits, noise = _logits(B, V, "bf16", rng), _noise(B, V, rng)
    lam = torch.full((1,), 0.5, device=DEV)
    par = dict(temperature=torch.full((B,), 0.8, device=DEV), top_k=_i32([50] * B),
               top_p=torch.tensor([1, 1, 0.9, 0.9, 0.99, 0.2], device=DEV), min_p=torch.zeros(B, device=DEV))

    def step():
        m = R.relation_page_map(cached, one, table, free, page, B)
        qr = R.relation_paged_append(k, v, kc, vc, m["slots"], m["positions"], q=q)
        y = R.relation_paged_decode(qr, kc, vc, table, m["lengths"], lam)
        return y["o"], y["row_stat"], *R.relation_sample(logits, noise, **par).values(), m["slots"], m["counts"]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for r in range(3):
        cached.copy_(_i32(rng.choice([1, 2, 31, 47, 250, 601], B)))
        for t in (q, k, v):
            t.normal_()
        noise.exponential_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b), r
