"""Refusals of the chunk step, the norms of heads and the log-probabilities, on the host: no GPU is needed, nothing is
launched."""
import ctypes
import math
import os

import pytest

from paper_2608_20172_amd import binding as R

BASE, MB = 0x7F0000000000, 1 << 24
BAD, UNSUP, WS, HIP, OK = (R.REL_ERR_INVALID_ARG, R.REL_ERR_UNSUPPORTED, R.REL_ERR_WORKSPACE, R.REL_ERR_HIP, R.REL_OK)
A = [BASE + i * MB for i in range(20)]


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(R.LIB_PATH):
        from paper_2608_20172_amd import build
        build.build()
    return R.load_library()


@pytest.fixture(autouse=True)
def _no_launch(monkeypatch):
    """The addresses here are made up: a call whose arguments are accepted ends right before its launch, also where
    there is a GPU."""
    monkeypatch.setenv("RELATION_TEST_FAIL_LAUNCH", "1")


# ---------------------------------------------------------------------------
def pages(P=100, page=16, H=2, D=64, dtype=R.REL_BF16, sp=None, sh=None, st=None):
    st = D if st is None else st
    sh = page * st if sh is None else sh
    return R.RelPages(P, page, H, D, dtype, H * sh if sp is None else sp, sh, st)


def chunk(lib, c=None, N=40, B=3, Hq=4, W=40, top=0, tau=2.0, scale=0.0, ws_bytes=1 << 23, **kw):
    a = {n: A[i] for i, n in enumerate("q kc vc table lengths start lam out stat ws".split())}
    a.update(kw)
    c = pages() if c is None else c
    d = R.RelPagedChunk(N, B, Hq, W, top, tau, scale)
    return lib.relation_paged_prefill(ctypes.byref(c), ctypes.byref(d), a["q"], a["kc"], a["vc"], a["table"], a["lengths"],
                                      a["start"], a["lam"], a["out"], a["stat"], a["ws"], ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(), HIP), (dict(N=0), OK), (dict(B=0), OK), (dict(Hq=0), OK), (dict(N=-1), BAD), (dict(B=-1), BAD), (dict(Hq=-2), BAD),
    (dict(Hq=3), BAD), (dict(W=0), BAD), (dict(W=1 << 27), UNSUP), (dict(B=4097), UNSUP), (dict(B=4096), HIP),
    (dict(N=(1 << 26) + 1), UNSUP), (dict(N=1 << 26, Hq=32), UNSUP), (dict(tau=0.0), BAD), (dict(tau=math.nan), BAD),
    (dict(scale=math.inf), BAD), (dict(scale=-1.0), HIP), (dict(top=10), HIP), (dict(N=1 << 62), UNSUP),
])
def test_chunk_sizes(lib, kw, code):
    assert chunk(lib, **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(P=-1), BAD), (dict(page=12), UNSUP), (dict(D=136), UNSUP), (dict(D=60), UNSUP), (dict(dtype=3), UNSUP),
    (dict(sh=-8), BAD), (dict(st=68), BAD), (dict(sp=64), BAD), (dict(st=32), BAD), (dict(P=0), BAD), (dict(H=0), BAD),
    (dict(st=1 << 30), UNSUP), (dict(D=120), HIP), (dict(D=4, dtype=R.REL_F32), HIP), (dict(sh=64, st=128, sp=2048), HIP),
])
def test_chunk_pool(lib, kw, code):
    assert chunk(lib, pages(**kw)) == code


def test_chunk_requests_times_heads(lib):
    """A grid of over 2^32 threads is refused."""
    for H, code in ((1024, HIP), (1025, UNSUP)):
        assert chunk(lib, c=pages(P=1, page=1, H=H, D=8), B=4096, Hq=H) == code


def test_chunk_pointers(lib):
    for n in ("q", "kc", "vc", "table", "lengths", "start", "lam", "out"):
        assert chunk(lib, **{n: None}) == BAD and chunk(lib, **{n: A[12] + 2}) == BAD
    for n in ("q", "kc", "vc", "out"):
        assert chunk(lib, **{n: A[12] + 8}) == BAD
    assert chunk(lib, stat=None) == HIP and chunk(lib, stat=A[12] + 2) == BAD
    for n in ("kc", "vc", "table", "lengths", "start", "lam", "q"):
        assert chunk(lib, out=A["q kc vc table lengths start lam".split().index(n)]) == BAD
        assert b"overlaps" in lib.relation_last_error()
    assert chunk(lib, stat=A[7]) == BAD and chunk(lib, vc=A[1]) == HIP  # keys as values: both are read
    d = R.RelPagedChunk(40, 3, 4, 40, 0, 2.0, 0.0)
    c = pages()
    need = lib.relation_paged_prefill_workspace_bytes(ctypes.byref(c), ctypes.byref(d))
    if need:
        assert chunk(lib, ws_bytes=need - 1) == WS and chunk(lib, ws=None) == WS and chunk(lib, ws=A[12] + 8) == BAD
        assert chunk(lib, ws=A[7]) == BAD
    assert lib.relation_paged_prefill_workspace_bytes(ctypes.byref(c), None) == 0
    assert lib.relation_paged_prefill(None, ctypes.byref(d), *A[:10], 1 << 23, None) == BAD
    assert lib.relation_paged_prefill(ctypes.byref(c), None, *A[:10], 1 << 23, None) == BAD


def test_chunk_workspace_over_the_range(lib):
    """The size grows with nothing but the sizes, and is 0 for what is refused."""
    for H, G, D in ((1, 1, 64), (8, 1, 64), (4, 4, 128), (12, 1, 32)):
        for N in (1, 17, 500, 20000):
            for W in (1, 8, 2048, 65536):
                c, d = pages(H=H, D=D), R.RelPagedChunk(N, min(N, 5), H * G, W, 0, 2.0, 0.0)
                need = lib.relation_paged_prefill_workspace_bytes(ctypes.byref(c), ctypes.byref(d))
                assert need % 4 == 0 and need < 1 << 34
                assert chunk(lib, c, N=N, B=min(N, 5), Hq=H * G, W=W, ws_bytes=need, kc=A[1], vc=A[2], out=A[9] + (1 << 40),
                             stat=A[9] + (1 << 41), ws=A[9] + (1 << 42), q=A[9] + (1 << 39)) == HIP
    assert lib.relation_paged_prefill_workspace_bytes(ctypes.byref(pages(D=60)), ctypes.byref(R.RelPagedChunk(4, 1, 2, 9, 0, 2.0, 0.0))) == 0


# ---------------------------------------------------------------------------
def norm_problem(B=2, T=10, Hq=4, H=2, D=64, dtype=R.REL_BF16, wdtype=R.REL_F32, norm=1, layout=0, eps=1e-6, amp=1.0, rope=64,
                 base=1e4, factor=1.0, length=0, low=1.0, high=32.0, pstride=10, **strides):
    q, k = (R.RelStrides(h * T * D, T * D, D) for h in (Hq, H))
    s = {"q": q, "k": k, "q_out": q, "k_out": k, "dq": q, "dk": k} | {n: R.RelStrides(*x) for n, x in strides.items()}
    return R.RelQkNorm(B, T, Hq, H, D, s["q"], s["k"], s["q_out"], s["k_out"], s["dq"], s["dk"], pstride, rope, length, base,
                       factor, low, high, dtype, wdtype, norm, layout, eps, amp)


def norm_fwd(lib, p=None, **kw):
    a = {n: A[i] for i, n in enumerate("q k wq wk pos qo ko".split())}
    a.update(kw)
    p = norm_problem() if p is None else p
    return lib.relation_qk_norm_fwd(ctypes.byref(p), *(a[n] for n in "q k wq wk pos qo ko".split()), None)


def norm_bwd(lib, p=None, ws_bytes=1 << 23, **kw):
    names = "q k wq wk pos gq gk dq dk dwq dwk ws".split()
    a = {n: A[i] for i, n in enumerate(names)}
    a.update(kw)
    p = norm_problem() if p is None else p
    return lib.relation_qk_norm_bwd(ctypes.byref(p), *(a[n] for n in names), ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(), HIP), (dict(B=0), OK), (dict(T=0), OK), (dict(Hq=0, H=0), OK), (dict(B=-1), BAD), (dict(T=-1), BAD), (dict(H=-1), BAD),
    (dict(D=0, rope=0), UNSUP), (dict(D=129), UNSUP), (dict(D=1, rope=0), HIP), (dict(D=63, rope=62), HIP), (dict(dtype=2), UNSUP),
    (dict(wdtype=7), UNSUP), (dict(norm=2), BAD), (dict(eps=0.0), BAD), (dict(eps=-1.0), BAD), (dict(eps=math.inf), BAD),
    (dict(eps=0.0, norm=0), HIP), (dict(rope=66), BAD), (dict(rope=31), BAD), (dict(rope=-2), BAD), (dict(layout=2), BAD),
    (dict(layout=2, rope=0), HIP), (dict(base=1.0), BAD), (dict(base=math.nan), BAD), (dict(factor=0.9), BAD), (dict(factor=math.inf), BAD),
    (dict(length=-1), BAD), (dict(low=2.0, high=2.0), BAD), (dict(low=math.nan), BAD), (dict(amp=math.nan), BAD), (dict(pstride=9), BAD),
    (dict(pstride=0), HIP), (dict(pstride=-1), BAD), (dict(pstride=1 << 41), UNSUP), (dict(B=1, pstride=3), HIP), (dict(H=1 << 17), UNSUP),
    (dict(B=1 << 16, T=1 << 16), UNSUP), (dict(q=(-1, 64, 64)), BAD), (dict(q=(0, 0, 0)), HIP), (dict(q_out=(0, 640, 64)), BAD),
    (dict(q_out=(2560, 640, 63)), BAD), (dict(k=(1 << 41, 64, 64)), UNSUP), (dict(k_out=(1 << 40, 1 << 38, 64)), HIP),
    (dict(Hq=0), HIP), (dict(H=0), HIP), (dict(B=1, T=(1 << 26) + 1), UNSUP),
])
def test_norm_sizes(lib, kw, code):
    far = dict(qo=A[9], ko=A[9] + (1 << 43))
    assert norm_fwd(lib, norm_problem(**kw), **far) == code


def test_norm_pointers(lib):
    for n in ("q", "k", "qo", "ko"):
        assert norm_fwd(lib, **{n: None}) == BAD and norm_fwd(lib, **{n: A[12] + 1}) == BAD
        assert norm_fwd(lib, **{n: A[12] + 2}) == HIP  # any element
    for n in ("wq", "wk", "pos"):
        assert norm_fwd(lib, **{n: None}) == HIP and norm_fwd(lib, **{n: A[12] + 2}) == BAD
    for n in ("q", "k", "wq", "wk", "pos", "ko"):
        at = A["q k wq wk pos qo ko".split().index(n)]
        assert norm_fwd(lib, qo=at) == BAD and b"overlaps" in lib.relation_last_error()
    assert norm_fwd(lib, k=A[0], wk=A[2]) == HIP  # inputs may be one
    assert norm_fwd(lib, norm_problem(Hq=0), q=None, qo=None) == HIP and norm_fwd(lib, norm_problem(H=0), k=None, ko=None) == HIP
    # slices of one [B, T, heads, D] buffer: apart by the query heads, or not
    s = (10 * 6 * 64, 64, 6 * 64)
    p = norm_problem(q_out=s, k_out=s)
    assert norm_fwd(lib, p, ko=A[5] + 4 * 64 * 2) == HIP and norm_fwd(lib, p, ko=A[5] + 3 * 64 * 2) == BAD
    assert norm_fwd(lib, p, ko=A[5] + 4 * 64 * 2 - 2) == BAD
    assert lib.relation_qk_norm_fwd(None, *A[:7], None) == BAD


def test_norm_backward(lib):
    assert norm_bwd(lib) == HIP
    for n in ("q", "k", "gq", "gk", "dq", "dk"):
        assert norm_bwd(lib, **{n: None}) == BAD and norm_bwd(lib, **{n: A[14] + 1}) == BAD
    for n in ("dwq", "dwk", "pos", "wq", "wk"):
        assert norm_bwd(lib, **{n: None}) == HIP and norm_bwd(lib, **{n: A[14] + 2}) == BAD
    p = norm_problem()
    need = lib.relation_qk_norm_bwd_workspace_bytes(ctypes.byref(p))
    assert need == 2 * 20 * 64 * 4
    assert norm_bwd(lib, ws_bytes=need) == HIP and norm_bwd(lib, ws_bytes=need - 1) == WS and norm_bwd(lib, ws=None) == WS
    assert norm_bwd(lib, ws=None, ws_bytes=0, dwq=None, dwk=None) == HIP and norm_bwd(lib, ws=A[14] + 8) == BAD
    for n, at in (("dq", 0), ("dk", 5), ("dq", 8), ("dwq", 1), ("dwk", 9), ("ws", 7), ("ws", 10), ("dk", 4)):
        assert norm_bwd(lib, **{n: A[at]}) == BAD, (n, at)
    no = norm_problem(norm=0)
    assert norm_bwd(lib, no) == BAD and norm_bwd(lib, no, dwq=None, dwk=None, ws=None) == HIP
    assert lib.relation_qk_norm_bwd_workspace_bytes(ctypes.byref(no)) == 0
    assert norm_bwd(lib, norm_problem(T=0, pstride=0)) == HIP  # the weights' gradients are still written, as zeros
    assert norm_bwd(lib, norm_problem(T=0, pstride=0), dwq=None, dwk=None) == OK
    assert norm_bwd(lib, norm_problem(dq=(0, 0, 0))) == BAD and norm_bwd(lib, norm_problem(q_out=(0, 0, 0), k_out=(0, 0, 0))) == HIP
    assert lib.relation_qk_norm_bwd(None, *A[:12], 0, None) == BAD


# ---------------------------------------------------------------------------
def score(lib, N=4, V=1000, K=5, dtype=R.REL_BF16, sl=1000, ws_bytes=1 << 23, **kw):
    names = "x t lp H rank tt tl stats ws".split()
    a = {n: A[i] for i, n in enumerate(names)}
    a.update(kw)
    p = R.RelTokenLogprobs(N, V, K, dtype, sl, 0)
    return lib.relation_token_logprobs_fwd(ctypes.byref(p), *(a[n] for n in names), ws_bytes, None)


def grad(lib, N=4, V=1000, dtype=R.REL_BF16, sl=1000, sg=1000, **kw):
    names = "x t stats g h d".split()
    a = {n: A[i] for i, n in enumerate(names)}
    a.update(kw)
    p = R.RelTokenLogprobs(N, V, 0, dtype, sl, sg)
    return lib.relation_token_logprobs_bwd(ctypes.byref(p), *(a[n] for n in names), None)


@pytest.mark.parametrize("kw,code", [
    (dict(), HIP), (dict(N=0), OK), (dict(N=-1), BAD), (dict(V=0), BAD), (dict(V=-1), BAD), (dict(K=-1), BAD), (dict(K=33), UNSUP),
    (dict(K=32), HIP), (dict(V=4, K=5), BAD), (dict(V=5), HIP), (dict(dtype=2), UNSUP), (dict(V=(1 << 22) + 1), UNSUP),
    (dict(N=(1 << 20) + 1), UNSUP), (dict(N=1 << 20, V=1 << 17, sl=1 << 17), UNSUP), (dict(sl=999), BAD), (dict(sl=0), HIP),
    (dict(sl=-1000), BAD), (dict(N=1, sl=-5), HIP), (dict(sl=1 << 41), UNSUP),
])
def test_score_sizes(lib, kw, code):
    assert score(lib, **kw) == code


def test_score_pointers(lib):
    for n in ("x", "t", "tt", "tl"):
        assert score(lib, **{n: None}) == BAD
    for n in ("lp", "H", "rank", "stats"):
        assert score(lib, **{n: None}) == HIP
    for n in ("x", "t", "lp", "H", "rank", "tt", "tl", "stats"):
        assert score(lib, **{n: A[12] + 1}) == BAD
    assert score(lib, stats=A[12] + 4) == BAD and score(lib, t=A[12] + 4) == BAD and score(lib, x=A[12] + 2) == HIP
    assert score(lib, K=0, tt=None, tl=None) == HIP
    for n in ("lp", "H", "rank", "tt", "tl", "stats"):
        assert score(lib, **{n: A[0] + 64}) == BAD and score(lib, **{n: A[1]}) == BAD
    assert score(lib, H=A[2]) == BAD
    p = R.RelTokenLogprobs(4, 200000, 5, R.REL_F32, 200000, 0)
    need = lib.relation_token_logprobs_workspace_bytes(ctypes.byref(p))
    big = dict(V=200000, dtype=R.REL_F32, sl=200000)
    assert need > 0 and score(lib, **big, ws_bytes=need) == HIP and score(lib, **big, ws_bytes=need - 1) == WS
    assert score(lib, **big, ws=None) == WS and score(lib, **big, ws=A[8] + 8) == BAD and score(lib, **big, ws=A[0]) == BAD
    assert lib.relation_token_logprobs_workspace_bytes(None) == 0
    assert lib.relation_token_logprobs_fwd(None, *A[:9], 0, None) == BAD


@pytest.mark.parametrize("kw,code", [
    (dict(), HIP), (dict(N=0), OK), (dict(V=0), BAD), (dict(sg=999), BAD), (dict(sg=0), BAD), (dict(N=1, sg=0), HIP), (dict(sl=0), HIP),
    (dict(sg=1 << 41), UNSUP), (dict(g=None), HIP), (dict(h=None), HIP), (dict(x=None), BAD), (dict(t=None), BAD), (dict(stats=None), BAD),
    (dict(d=None), BAD), (dict(stats=A[9] + 8), BAD), (dict(d=A[9] + 1), BAD), (dict(d=A[9] + 2), HIP), (dict(d=A[0]), BAD),
    (dict(d=A[2]), BAD), (dict(d=A[3] - 4), BAD), (dict(g=A[9] + 2), BAD), (dict(x=A[9] + 1), BAD),
])
def test_gradient(lib, kw, code):
    assert grad(lib, **kw) == code
