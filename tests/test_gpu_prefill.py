"""GPU parity of chunks of new tokens over a paged cache with the fp64 serving oracle.

Bars, all relative l2. M: fp32 arithmetic, 2e-5 (exponents reach 40, an fp32 rounding of them 4e-6). y in fp32: the
same. y in bf16: one rounding of the weights and one of y, each at most 2^-8 of what it rounds; the weights' errors add
up like the weighted values themselves, so 2 * 2^-8."""
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
BAR = {"bf16": 2.0 ** -7, "f32": 2e-5}
BAR_M = 2e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    R.load_library()


def _np(t):
    return t.detach().double().cpu().numpy()


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _rows(rng, shape, dtype, std=1.0):
    return torch.from_numpy(rng.standard_normal(shape) * std).to(TORCH_DT[dtype]).to(DEV)


def _step(chunks, H, G, D, page, dtype, layout="hnd", seed=0, std=1.0, junk=math.nan):
    """A step of requests (cached, added): what the call takes. Entries of no request hold `junk`."""
    rng = np.random.default_rng(seed + D + page)
    lens = [c + n for c, n in chunks]
    used = [-(-n // page) for n in lens]
    W, pages = max(1, max(used)), sum(used) + 2
    ids, table, at = rng.permutation(pages), np.full((len(lens), W), -1), 0
    for b, n in enumerate(used):
        table[b, :n] = ids[at:at + n]
        at += n
    shape = (2, pages, page, H, D) if layout == "nhd" else (2, pages, H, page, D)
    x = _rows(rng, shape, dtype)
    if layout == "joint":  # both pools in one allocation
        both = torch.stack([x[0], x[1]], 1).contiguous()
        kc, vc = both[:, 0], both[:, 1]
    elif layout == "wide":  # rows 64 elements apart
        y = torch.zeros(shape[:-1] + (D + 64,), dtype=x.dtype, device=DEV)
        y[..., :D] = x
        kc, vc = y[0][..., :D], y[1][..., :D]
    else:
        kc, vc = (t.transpose(1, 2) if layout == "nhd" else t for t in x)
    kc *= std
    free = np.ones((pages, page), bool)
    for b, n in enumerate(lens):
        for j in range(n):
            free[table[b, j // page], j % page] = False
    mask = torch.tensor(free, device=DEV)[:, None, :, None]
    kc.masked_fill_(mask, junk)
    vc.masked_fill_(mask, junk)
    start = np.concatenate([[0], np.cumsum([n for _, n in chunks])])
    q = _rows(rng, (int(start[-1]), H * G, D), dtype, std)
    return {"q": q, "kc": kc, "vc": vc, "table": table, "lens": np.array(lens), "start": start}


def _run(s, lam=0.4, **kw):
    r = R.relation_paged_prefill(s["q"], s["kc"], s["vc"], _i32(s["table"]), _i32(s["lens"]), _i32(s["start"]), lam, **kw)
    torch.cuda.synchronize()
    return r


def _close(r, s, dtype, lam=0.4, most=40, **kw):
    """Against the oracle, at up to `most` rows a request: its first and last ones, and some between."""
    rows = set()
    for a, e in zip(s["start"][:-1], s["start"][1:]):
        rows |= set(range(a, min(e, a + 3))) | set(range(max(a, e - 3), e))
        rows |= set(np.linspace(a, max(a, e - 1), max(1, most // max(1, len(s["lens"])))).astype(int).tolist()) if e > a else set()
    Y, M = SO.paged_prefill(_np(s["q"]), _np(s["kc"]), _np(s["vc"]), s["table"], s["lens"], s["start"], float(np.float32(lam)),
                            rows=rows, **kw)
    rows = sorted(rows)
    Y, M = np.stack([Y[x] for x in rows]), np.stack([M[x] for x in rows])
    y, m = _np(r["o"])[rows], _np(r["row_stat"])[rows]
    assert np.array_equal(np.isnan(y), np.isnan(Y)) and np.array_equal(np.isnan(m), np.isnan(M))
    ok = ~np.isnan(M)
    ey, em = rel_l2(y[ok], Y[ok]), rel_l2(m[ok], M[ok])
    log(f"  y: rel-l2 {ey:.2e} (bar {BAR[dtype]:.1e}); M: {em:.2e} (bar {BAR_M:.1e}); {len(rows)} rows")
    assert ey <= BAR[dtype] and em <= BAR_M


@pytest.mark.parametrize("chunks,H,G,D,page,dtype,layout", [
    ([(0, 1)], 1, 1, 64, 16, "bf16", "hnd"), ([(1, 1)], 8, 1, 64, 16, "bf16", "nhd"), ([(0, 2)], 2, 3, 32, 1, "bf16", "hnd"),
    ([(0, 1), (1, 1), (2, 3), (15, 2), (16, 17)], 2, 2, 32, 16, "bf16", "hnd"),
    ([(0, 128), (0, 129), (0, 63), (0, 64), (0, 65)], 2, 1, 64, 16, "bf16", "hnd"),
    ([(200, 24)], 8, 1, 64, 16, "bf16", "hnd"), ([(700, 5), (5, 700), (1, 1)], 3, 4, 80, 8, "bf16", "nhd"),
    ([(1025, 33), (33, 0), (0, 40)], 2, 3, 96, 32, "bf16", "joint"), ([(0, 300)], 1, 8, 128, 64, "bf16", "hnd"),
    ([(290, 31)], 2, 5, 48, 1, "bf16", "wide"), ([(0, 301), (777, 150), (41, 41)], 4, 1, 80, 16, "f32", "hnd"),
    ([(257, 1), (100, 99)], 2, 4, 128, 128, "f32", "nhd"), ([(0, 77)], 1, 3, 4, 16, "f32", "hnd"),
    ([(40, 1), (1, 0), (9, 9)], 2, 7, 8, 4, "bf16", "hnd"), ([(3000, 2)], 2, 1, 64, 512, "bf16", "nhd"),
    ([(2100, 17), (17, 400)], 1, 6, 128, 16, "bf16", "joint"), ([(1000, 100), (2999, 1)], 2, 2, 128, 1024, "f32", "hnd"),
    ([(60, 1)] * 40 + [(3, 2)] * 30, 3, 1, 64, 16, "bf16", "hnd"), ([(130, 1)] * 20, 2, 16, 64, 16, "bf16", "hnd"),
    ([(0, 200), (90, 9)], 1, 130, 112, 16, "bf16", "nhd"), ([(50, 20)], 2, 12, 120, 16, "f32", "hnd"),
    ([(0, 90)], 2, 1, 32, 16, "f32", "nhd"), ([(0, 500), (64, 64)], 2, 1, 60 // 4 * 4, 2, "f32", "hnd"),
    ([(0, 1000)], 12, 1, 64, 16, "bf16", "nhd"), ([(5, 0), (0, 0)], 2, 1, 64, 16, "bf16", "hnd"),
])
def test_prefill(chunks, H, G, D, page, dtype, layout):
    log(f"[prefill] {chunks[:5]} H={H} G={G} D={D} page={page} {dtype} {layout}")
    s = _step(chunks, H, G, D, page, dtype, layout)
    r = _run(s)
    if s["start"][-1]:
        _close(r, s, dtype)
    for b, (c, n) in enumerate(chunks):  # the first token of all: y is its own value exactly
        if c == 0 and n:
            assert torch.equal(r["o"][s["start"][b]], s["vc"][s["table"][b, 0], :, 0].repeat_interleave(G, 0))


def test_prefill_many_requests():
    """More requests than threads, some without tokens: the scan over the requests takes several of them a thread."""
    for B in (255, 256, 257, 1000):
        chunks = [(b % 37, (b * 7) % 4) for b in range(B)]
        log(f"[prefill] {B} requests")
        s = _step(chunks, 1, 2, 32, 8, "bf16")
        _close(_run(s), s, "bf16", most=1)


def test_prefill_of_4096_requests():
    """The largest batch; one more is refused."""
    chunks = [(b % 11, 1 + (b == 4000) * 200) for b in range(4096)]
    s = _step(chunks, 1, 1, 32, 16, "bf16")
    r = _run(s)
    part = {n: s[n] for n in ("q", "kc", "vc")} | {"table": s["table"][3990:4010], "lens": s["lens"][3990:4010],
                                                   "start": s["start"][3990:4011]}
    _close(r, part, "bf16")
    assert not torch.isnan(r["o"]).any()
    with pytest.raises(RuntimeError, match="requests"):
        R.relation_paged_prefill(s["q"], s["kc"], s["vc"], _i32(np.zeros((4097, 1))), _i32(np.ones(4097)), _i32(np.zeros(4098)), 0.4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("G", [1, 6])
def test_prefill_sharp(dtype, G):
    """Evidence of tens of units: rows whose totals pass 2^64 are scanned again; and scale, tau_s, lambda and max_length
    given."""
    s = _step([(640, 137), (0, 130), (60, 4)], 2, G, 64, 16, dtype, std=4.0)
    _close(_run(s, -0.7, max_length=777), s, dtype, -0.7, max_length=777)
    s = _step([(500, 100), (0, 130), (0, 1)], 2, G, 64, 16, dtype, std=1.5)
    _close(_run(s, 2.0, scale=0.3, tau_s=0.5, max_length=640), s, dtype, 2.0, scale=0.3, tau_s=0.5)


@pytest.mark.parametrize("chunks,H,G,D,page,dtype", [
    ([(5000, 40)], 2, 1, 64, 16, "bf16"), ([(9000, 3), (100, 200), (4097, 1)], 1, 4, 128, 32, "bf16"), ([(4200, 130)], 3, 2, 48, 8, "bf16"),
    ([(4400, 33), (5, 5)], 1, 3, 80, 16, "f32"), ([(6000, 1)] * 3, 2, 2, 120, 64, "f32"), ([(4700, 300)], 1, 1, 32, 1, "bf16"),
    ([(700, 20)], 1, 1, 4, 4, "f32"), ([(2500, 8), (1, 1)], 2, 1, 24, 16, "bf16"), ([(513, 1), (512, 1), (511, 2), (1024, 1)], 1, 1, 64, 16, "bf16"),
    ([(4500, 60)], 2, 1, 100, 16, "f32"), ([(8000, 1)] * 70, 1, 1, 32, 128, "bf16"),
])
def test_prefill_long_histories(chunks, H, G, D, page, dtype):
    """Few rows over many keys: the history in slices, joined by a second kernel; rows whose history ends in any slice."""
    log(f"[prefill] slices {chunks[:4]} H={H} G={G} D={D} page={page} {dtype}")
    s = _step(chunks, H, G, D, page, dtype)
    c, d = R.make_pages(s["kc"], s["vc"]), R.RelPagedChunk(s["q"].shape[0], len(chunks), H * G, s["table"].shape[1], 0, 2.0, 0.0)
    assert R.load_library().relation_paged_prefill_workspace_bytes(R.ctypes.byref(c), R.ctypes.byref(d)) > 0  # several slices
    r = _run(s)
    _close(r, s, dtype, most=12)
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device=DEV)  # states that nobody writes are NaN there
    again = _run(s, workspace=ws)
    assert torch.equal(r["o"], again["o"]) and torch.equal(r["row_stat"], again["row_stat"])


@pytest.mark.parametrize("dtype,D,G,n", [("bf16", 64, 1, 40), ("bf16", 128, 4, 50), ("f32", 80, 2, 3)])
def test_prefill_slices_that_are_scanned_again(dtype, D, G, n):
    """Totals past 2^64 in some slices, values that are not finite behind rows and in their history, and bad pages: in
    the slices where they are."""
    chunks = [(4600, n), (4300, 2)]
    s = _step(chunks, 2, G, D, 16, dtype, std=4.0)
    _close(_run(s), s, dtype, most=12)
    s = _step(chunks, 2, G, D, 16, dtype)
    base = _run(s)
    at = 4600 + n - 2  # the last row but one: it and the last row have the entry
    for value in (math.nan, math.inf):
        t = {**s, "vc": s["vc"].clone()}
        t["vc"][s["table"][0, at // 16], 1, at % 16, 3] = value
        r = _run(t)
        o, w = r["o"].view(-1, 2, G, D), base["o"].view(-1, 2, G, D)
        assert torch.equal(o[:, 0], w[:, 0]) and torch.equal(o[n:], w[n:])
        assert rel_l2(_np(o[:n - 2]), _np(w[:n - 2])) <= BAR[dtype] if n > 2 else True
        assert not torch.isfinite(o[n - 2:n, 1, :, 3]).any()
        t["vc"][s["table"][0, 100 // 16], 0, 100 % 16, 5] = value  # far back: all rows of the head
        r = _run(t)
        assert not torch.isfinite(r["o"].view(-1, 2, G, D)[:n, 0, :, 5]).any() and torch.isfinite(r["o"][n:]).all()
        assert torch.isfinite(r["row_stat"]).all()
    P = s["kc"].shape[0]
    t = {**s, "table": s["table"].copy()}
    t["table"][1, 10] = P
    if n > 8:  # the first row's page is the one before
        t["table"][0, 4600 // 16 + 1] = -1
    r = _run(t)
    _close(r, t, dtype, most=12)
    assert torch.isnan(r["row_stat"][n:]).all() and not torch.isnan(r["row_stat"][0]).any()


def test_prefill_is_decode_a_token_at_a_time():
    """Every row of the chunk as relation_paged_decode gives it at that length."""
    s = _step([(300, 40), (0, 23)], 4, 2, 64, 16, "bf16", "nhd")
    r = _run(s)
    for b in range(2):
        a, e = s["start"][b], s["start"][b + 1]
        n = e - a
        lens = s["lens"][b] - n + 1 + np.arange(n)
        d = R.relation_paged_decode(s["q"][a:e], s["kc"], s["vc"], _i32(np.repeat(s["table"][b][None], n, 0)), _i32(lens), 0.4)
        # bf16: the decode step's rows have one rounding of y, these two roundings
        ey, em = rel_l2(_np(r["o"][a:e]), _np(d["o"])), rel_l2(_np(r["row_stat"][a:e]), _np(d["row_stat"]))
        log(f"  request {b}: y {ey:.2e}, M {em:.2e}")
        assert ey <= 3 * 2.0 ** -8 and em <= 2 * BAR_M


def test_prefill_is_the_whole_sequence_whatever_the_chunks():
    """A prompt whole, in uneven parts and a token at a time: the rows of relation_fwd."""
    rng = np.random.default_rng(5)
    T, H, D, page = 333, 3, 64, 16
    q, k, v = (_rows(rng, (T, H, D), "bf16") for _ in range(3))
    kc, vc = (torch.zeros((30, H, page, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = rng.permutation(30)[None, :-(-T // page)]
    slots = torch.tensor([table[0, j // page] * page + j % page for j in range(T)], device=DEV)
    R.relation_paged_append(k, v, kc, vc, slots, _i32(np.arange(T)), rope_base=None)
    f = R.relation_fwd(*(x.transpose(0, 1)[None].contiguous() for x in (q, k, v)), 0.3)
    want, wm = f["o"][0].transpose(0, 1), f["row_stat"][0].transpose(0, 1)
    for parts in ([T], [1, 200, 100, 32], [150, 150, 33], [64] * 5 + [13]):
        got, gm, at = [], [], 0
        for n in parts:
            r = R.relation_paged_prefill(q[at:at + n], kc, vc, _i32(table), _i32([at + n]), _i32([0, n]), 0.3)
            got.append(r["o"])
            gm.append(r["row_stat"])
            at += n
        ey, em = rel_l2(_np(torch.cat(got)), _np(want)), rel_l2(_np(torch.cat(gm)), _np(wm))
        log(f"  parts {parts}: y {ey:.2e}, M {em:.2e}")
        assert ey <= 2 * BAR["bf16"] and em <= 2 * BAR_M  # two roundings on either side


@pytest.mark.parametrize("page", [1, 16, 128])
def test_prefill_shared_prefix(page):
    """Requests whose tables begin with the same pages."""
    s = _step([(256, 60), (256, 1), (256, 130)], 2, 2, 64, page, "bf16", "nhd")
    for b in (1, 2):
        s["table"][b, :256 // page] = s["table"][0, :256 // page]
    _close(_run(s), s, "bf16")


@pytest.mark.parametrize("G,n", [(1, 30), (4, 100)])
def test_prefill_bad_lengths_and_pages(G, n):
    """A request with a length under its tokens or over the bound is NaN, a row is NaN from the first bad page on, the
    others are as they are, and what the table holds past a length is not looked at."""
    chunks = [(20, n)] * 8
    s = _step(chunks, 2, G, 64, 16, "bf16")
    good = _run(s)
    s["lens"][[0, 1, 2, 3]] = [n - 1, -5, 10 ** 9, 0]
    P = s["kc"].shape[0]
    s["table"] = np.concatenate([s["table"], np.full((8, 3), -9)], 1)
    s["table"][4, 0], s["table"][5, 2], s["table"][6, (n + 19) // 16] = P, -1, 2 ** 31 - 1
    r = _run(s, max_length=n + 20)
    _close(r, s, "bf16", max_length=n + 20)
    lost = torch.isnan(r["row_stat"]).any(1).view(8, n)
    assert lost[:5].all() and not lost[7].any() and lost[5].any() and not lost[5].all() and lost[6].any()
    assert torch.equal(r["o"][-n:], good["o"][-n:])


@pytest.mark.parametrize("chunks", [[(100, 60)], [(0, 200)], [(90, 3), (0, 5)], [(300, 1)]])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype,D,G", [("bf16", 64, 1), ("bf16", 80, 4), ("f32", 64, 2)])
def test_prefill_what_is_behind_a_row_does_not_reach_it(chunks, value, dtype, D, G):
    """A value, and a key, that is not finite: the rows before it keep their bits, those after it are not finite."""
    s = _step(chunks, 2, G, D, 16, dtype)
    base = _run(s)
    for what in ("vc", "kc"):
        for back in (1, 2, 40, 70):  # entries from the end of the first request
            at = s["lens"][0] - back
            if at < 0:
                continue
            t = {**s, what: s[what].clone(memory_format=torch.preserve_format)}
            t[what][s["table"][0, at // 16], 1, at % 16, 5] = value
            r = _run(t)
            n = s["start"][1]
            first = max(0, at - (s["lens"][0] - n))  # the first row that has the entry
            o, w = r["o"].view(-1, 2, G, D), base["o"].view(-1, 2, G, D)
            assert torch.equal(o[:, 0], w[:, 0]) and torch.equal(o[n:], w[n:])
            near = rel_l2(_np(o[:first]), _np(w[:first])) if first else 0.0
            assert near <= BAR[dtype], near  # scanned again: other sums, the same rows
            assert not torch.isfinite(o[first:n, 1, :, 5]).any() or what == "kc"
            if what == "vc":
                rest = [d for d in range(D) if d != 5]
                assert rel_l2(_np(o[..., rest]), _np(w[..., rest])) <= BAR[dtype]
                assert rel_l2(_np(r["row_stat"]), _np(base["row_stat"])) <= BAR_M


def test_prefill_rows_of_no_request_are_left():
    s = _step([(10, 5), (0, 3)], 2, 1, 64, 16, "bf16")
    s["q"] = torch.cat([s["q"], s["q"]])
    o = torch.full_like(s["q"], 7.0)
    rs = torch.full((16, 2), 7.0, device=DEV)
    r = _run(s, out={"o": o, "row_stat": rs})
    assert r["o"] is o and bool((o[8:] == 7).all()) and bool((rs[8:] == 7).all()) and bool((rs[:8] != 7).all())
    t = {**s, "start": s["start"] + 4}  # and before the first
    o.fill_(7.0)
    _run(t, out={"o": o, "row_stat": rs.fill_(7.0)})
    assert bool((o[:4] == 7).all()) and bool((o[12:] == 7).all()) and bool((rs[4:12] != 7).all())


@pytest.mark.parametrize("start", [[0, 5, 3], [-7, 5, 8], [0, 5, 10 ** 9], [3, 3, 3], [8, 4, 0], [2 ** 31 - 1, -2 ** 31, 5]])
def test_prefill_any_row_start_stays_inside(start):
    """Starts that are not ascending or past the rows: nothing outside the buffers is touched (guards around out)."""
    s = _step([(10, 5), (0, 3)], 2, 1, 64, 16, "bf16")
    guard = torch.full((24, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    s["start"] = np.array(start)
    _run(s, out={"o": guard[8:16]})
    assert bool((guard[:8] == 7).all()) and bool((guard[16:] == 7).all())


def test_prefill_repeats_its_bits_on_a_stream_and_in_a_graph():
    s = _step([(300, 200), (7, 1), (0, 90)], 4, 2, 64, 16, "bf16")
    first = _run(s)
    a = [s["q"], s["kc"], s["vc"], _i32(s["table"]), _i32(s["lens"]), _i32(s["start"]), torch.full((1,), 0.4, device=DEV)]
    out = {"o": torch.empty_like(s["q"]), "row_stat": torch.empty_like(first["row_stat"])}
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        R.relation_paged_prefill(*a, out=out)
    stream.synchronize()
    assert torch.equal(out["o"], first["o"]) and torch.equal(out["row_stat"], first["row_stat"])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.relation_paged_prefill(*a, out=out)
    same = lambda x, y: torch.equal(x.isnan(), y.isnan()) and torch.equal(x.nan_to_num(), y.nan_to_num())
    for turn in range(4):  # other lengths and starts in the same buffers (past the second request's pages: NaN rows)
        chunks = [(300 - turn, 200 - 40 * turn), (7, 1 + 40 * turn), (0, 90)]
        lens, start = [c + n for c, n in chunks], np.concatenate([[0], np.cumsum([n for _, n in chunks])])
        a[4].copy_(_i32(lens))
        a[5].copy_(_i32(start))
        out["o"].zero_()
        graph.replay()
        torch.cuda.synchronize()
        want = R.relation_paged_prefill(*a)
        assert same(out["o"], want["o"]) and same(out["row_stat"], want["row_stat"])


def test_prefill_offsets_past_32_bits():
    """A pool of over 2^32 elements (9 GB in bf16), its last pages."""
    pages, H, page, D = 8200, 16, 256, 128
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 20 GB")
    kc, vc = (torch.zeros((pages, H, page, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    rng = np.random.default_rng(12)
    table, n = np.array([[8199, 8197]]), 300
    for x in (kc, vc):
        x[[8197, 8199]] = _rows(rng, (2, H, page, D), "bf16")
    q = _rows(rng, (40, H, D), "bf16")
    s = {"q": q, "kc": kc, "vc": vc, "table": table, "lens": np.array([n]), "start": np.array([0, 40])}
    r = _run(s)
    small = {**s, "kc": kc[[8197, 8199]], "vc": vc[[8197, 8199]], "table": np.array([[1, 0]])}
    del kc, vc, s
    _close(r, small, "bf16", most=8)
    torch.cuda.empty_cache()


def test_prefill_head_dim_and_shapes_are_checked():
    s = _step([(10, 5)], 2, 1, 64, 16, "bf16")
    for bad in (dict(head_dim=0), dict(head_dim=65), dict(head_dim=60, scale=0.1)):
        with pytest.raises(ValueError, match="head_dim"):
            _run(s, **bad)
    a, b = _run(s, head_dim=60), _run(s, scale=60 ** -0.5)
    assert torch.equal(a["o"], b["o"])
    for bad in (dict(start=np.array([0, 5, 5])), dict(lens=np.array([15, 3])), dict(table=s["table"][0]), dict(q=s["q"][..., :32]),
                dict(q=s["q"].float())):
        with pytest.raises((ValueError, RuntimeError)):
            _run({**s, **bad})
    with pytest.raises(ValueError, match="GPU"):
        R.relation_paged_prefill(s["q"].cpu(), s["kc"], s["vc"], _i32(s["table"]), _i32(s["lens"]), _i32(s["start"]), 0.4)


@pytest.mark.parametrize("B,G,H,long", [(64, 4, 2, 40), (65, 4, 2, 40), (64, 1, 1, 900), (63, 9, 1, 5), (33, 2, 2, 3000), (7, 1, 3, 4500),
                                        (64, 16, 8, 300)])
def test_prefill_every_tile_is_somebodys(B, G, H, long):
    """Requests of none, one, a tile's and many tokens behind histories of all lengths, in a shuffled order: every row is
    written, and by the right workgroup."""
    rng = np.random.default_rng(B + G + long)
    added = rng.choice([0, 1, 1, 1, 8, 32 // G, 33, 128 // G, 128 // G + 1, 200], B)
    chunks = [(int(c), int(n)) for c, n in zip(rng.integers(0, long, B), added)]
    log(f"[prefill] {B} requests, {sum(added)} tokens after up to {long}")
    s = _step(chunks, H, G, 32, 16, "bf16")
    out = {"o": torch.full_like(s["q"], math.inf), "row_stat": torch.full((s["q"].shape[0], H * G), math.inf, device=DEV)}
    r = _run(s, out=out)
    assert torch.isfinite(r["o"]).all() and torch.isfinite(r["row_stat"]).all()
    _close(r, s, "bf16", most=B)


@pytest.mark.parametrize("chunks", [[(100, 60), (0, 40)], [(90, 3), (0, 5)], [(5000, 30)]])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_prefill_a_query_that_is_not_finite_spoils_its_row_alone(chunks, value):
    s = _step(chunks, 2, 2, 64, 16, "bf16")
    base = _run(s)
    t = {**s, "q": s["q"].clone()}
    t["q"][1, 3, 7] = value
    r = _run(t)
    assert not torch.isfinite(r["o"][1, 3]).any() or value == math.inf  # infinite evidence of either sign may leave a row
    o, w = r["o"].clone(), base["o"].clone()
    o[1, 3], w[1, 3] = 0, 0
    assert rel_l2(_np(o), _np(w)) <= BAR["bf16"] and torch.equal(o[:, :2], w[:, :2])
    m, n = r["row_stat"].clone(), base["row_stat"].clone()
    m[1, 3] = n[1, 3] = 0
    assert rel_l2(_np(m), _np(n)) <= BAR_M


@pytest.mark.parametrize("B,H,D,n,dtype", [(3, 8, 64, 1500, "bf16"), (1, 8, 128, 3000, "bf16"), (40, 8, 64, 80, "bf16"), (3, 8, 80, 700, "f32"),
                                           (33, 8, 64, 1, "bf16"), (5, 16, 32, 900, "bf16")])
def test_prefill_sizes_between_few_and_many_tiles(B, H, D, n, dtype):
    """Fresh and cached chunks where the rule for a tile's rows changes."""
    chunks = [((b * 131) % 400, max(1, n - 17 * b)) for b in range(B)]
    s = _step(chunks, H, 1, D, 16, dtype)
    _close(_run(s), s, dtype, most=24)


@pytest.mark.parametrize("chunks,H,G,D", [
    ([(200, 1), (40, 1), (700, 1)], 2, 1, 64), ([(1000, 1)] * 20, 4, 4, 128), ([(333, 20)], 8, 1, 64), ([(5000, 3)], 2, 2, 96),
    ([(2000, 1)] * 8 + [(100, 130)] * 4, 4, 4, 128), ([(9000, 1)], 1, 32, 80),
])
@pytest.mark.parametrize("again", [False, True])
def test_prefill_weights_of_few_rows_are_as_the_decode_steps(chunks, H, G, D, again):
    """Where a request has at most 32 rows of a key head, its weights are as exact as the decode step's: with all
    values 1 the row is their sum over itself, 1 to 2^-16 for weights of 16 significant bits, so 1 in bf16; with equal keys the
    rounding of a weight to 8 bits would stand there whole. again: totals over 2^62, which are summed a second time."""
    rng = np.random.default_rng(len(chunks))
    s = _step(chunks, H, G, D, 16, "bf16")
    s["vc"].fill_(1.0)
    s["kc"].fill_(0.25)
    # U = scale sum(q) / 4, another for every row, from 2 on; or from 60
    N = int(s["start"][-1])
    u = torch.from_numpy(rng.random((N, H * G, 1)) * 6 + (60 if again else 2)).to(DEV)
    s["q"] = (u * 4 / math.sqrt(D) * torch.ones(D, device=DEV)).to(torch.bfloat16)
    r = _run(s)
    for b, (c, n) in enumerate(chunks):
        if n * G > 32:
            continue
        at = slice(int(s["start"][b]), int(s["start"][b + 1]))
        assert bool((r["o"][at] == 1).all()), (b, float((r["o"][at].float() - 1).abs().max()))
    one = [b for b, (c, n) in enumerate(chunks) if n == 1]
    if one:
        at = torch.tensor([int(s["start"][b]) for b in one], device=DEV)
        d = R.relation_paged_decode(s["q"][at], s["kc"], s["vc"], _i32(s["table"][one]), _i32(s["lens"][one]), 0.4)
        assert bool((d["o"] == 1).all())


@pytest.mark.parametrize("chunks,H,G,D,dtype", [
    ([(201, 24)], 8, 1, 64, "bf16"), ([(0, 300), (500, 1), (0, 1), (70, 3)], 2, 4, 128, "bf16"), ([(0, 700)], 2, 1, 64, "bf16"),
    ([(100, 60), (9, 0), (0, 33)], 2, 2, 80, "f32"),
])
def test_prefill_table_wider_than_the_requests(chunks, H, G, D, dtype):
    """A table of 32768 tokens a request, as a serving loop keeps for its longest context: tiles and slices go by it, most
    slices have no keys. With max_length and without, against the oracle."""
    s = _step(chunks, H, G, D, 16, dtype)
    wide = np.full((len(chunks), 2048), -1)
    wide[:, :s["table"].shape[1]] = s["table"]
    s["table"] = wide
    for kw in ({}, {"max_length": int(max(s["lens"]))}, {"max_length": 5000}):
        r = _run(s, **kw)
        _close(r, s, dtype)
        assert not torch.isnan(r["o"]).any()
