"""Refusals of the serving entry points, on the host: no GPU is needed, nothing is launched."""
import ctypes
import os

import pytest
import torch

from paper_2608_20172_amd import binding as R

BASE, MB = 0x7F0000000000, 1 << 24
BAD, UNSUP, WS, HIP, OK = (R.REL_ERR_INVALID_ARG, R.REL_ERR_UNSUPPORTED, R.REL_ERR_WORKSPACE, R.REL_ERR_HIP, R.REL_OK)
A = [BASE + i * MB for i in range(16)]


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


def pages(P=10, page=16, H=2, D=64, dtype=R.REL_BF16, sp=None, sh=None, st=None):
    st = D if st is None else st
    sh = page * st if sh is None else sh
    return R.RelPages(P, page, H, D, dtype, H * sh if sp is None else sp, sh, st)


# ---------------------------------------------------------------------------
def page_map(lib, m=(4, 8, 16, 100, 50), **kw):
    a = {n: A[i] for i, n in enumerate("cached added free table lengths start slots positions counts".split())}
    a.update(kw)
    d = R.RelPageMap(*m) if m else None
    return lib.relation_page_map(ctypes.byref(d) if d else None, a["cached"], a["added"], a["free"], a["table"],
                                 a["lengths"], a["start"], a["slots"], a["positions"], a["counts"], None)


@pytest.mark.parametrize("m,code", [
    ((4, 8, 16, 100, 50), HIP), (None, BAD), ((-1, 8, 16, 100, 50), BAD), ((4, -8, 16, 100, 50), BAD),
    ((4, 8, 16, -1, 50), BAD), ((4, 8, 16, 100, -1), BAD), ((4, 8, 24, 100, 50), UNSUP), ((4, 8, 0, 100, 50), UNSUP),
    ((4, 8, 1 << 17, 100, 50), UNSUP), ((4, 0, 16, 100, 50), BAD), ((4097, 8, 16, 100, 50), UNSUP),
    ((4, 1 << 27, 16, 100, 50), UNSUP), ((4, 1 << 62, 16, 100, 50), UNSUP), ((4, 8, 16, 1 << 31, 50), UNSUP),
    ((4, 8, 16, 100, 1 << 31), UNSUP), ((4096, 8, 16, 0, 0), HIP),
])
def test_page_map_sizes(lib, m, code):
    assert page_map(lib, m) == code


def test_page_map_pointers(lib):
    for n in ("cached", "added", "free", "table", "lengths", "start", "slots", "positions", "counts"):
        assert page_map(lib, **{n: None}) == BAD
        assert page_map(lib, **{n: A[12] + 2}) == BAD
    assert page_map(lib, slots=A[12] + 4) == BAD                       # 8-byte entries
    assert page_map(lib, (4, 8, 16, 0, 0), slots=None, positions=None, free=None) == HIP
    for n in ("table", "lengths", "slots", "counts"):
        assert page_map(lib, **{n: A[0]}) == BAD                       # over cached
    assert page_map(lib, lengths=A[3] + 4 * 8 * 4 - 4) == BAD          # inside the table's last entry
    assert page_map(lib, lengths=A[3] + 4 * 8 * 4) == HIP
    assert b"overlaps" in lib.relation_last_error() or page_map(lib, counts=A[0]) == BAD


# ---------------------------------------------------------------------------
def append(lib, c=None, N=5, Hq=2, D=64, s=(128, 64, 128, 64), rope=1e4, givens=1, **kw):
    a = {n: A[i] for i, n in enumerate("q k v slots positions theta qo kc vc".split())}
    a.update(kw)
    c = pages() if c is None else c
    n = R.RelAppend(N, Hq, D, *s, rope, givens)
    return lib.relation_paged_append(ctypes.byref(c), ctypes.byref(n), a["q"], a["k"], a["v"], a["slots"], a["positions"],
                                     a["theta"], a["qo"], a["kc"], a["vc"], None)


POOLS = [
    (dict(), HIP), (dict(P=-1), BAD), (dict(page=12), UNSUP), (dict(page=1 << 17), UNSUP), (dict(D=136), UNSUP),
    (dict(D=60), UNSUP), (dict(D=0), UNSUP), (dict(dtype=3), UNSUP), (dict(sh=-8), BAD), (dict(st=68), BAD),
    (dict(sp=64), BAD), (dict(st=32), BAD), (dict(P=1 << 29), UNSUP), (dict(H=1 << 17), UNSUP),
    (dict(st=1 << 30), UNSUP), (dict(sp=1 << 33), UNSUP), (dict(sh=64, st=128, sp=2048), HIP), (dict(P=0), BAD), (dict(H=0), BAD),
]


@pytest.mark.parametrize("c,code", POOLS)
def test_append_pool(lib, c, code):
    assert append(lib, pages(**c)) == code


def test_append_arguments(lib):
    assert append(lib, N=0) == OK and append(lib, N=-1) == BAD and append(lib, N=1 << 27) == UNSUP
    assert append(lib, D=65) == BAD and append(lib, D=0) == BAD and append(lib, D=63) == BAD
    assert append(lib, D=63, rope=0.0) == HIP and append(lib, D=10) == HIP
    for rope in (0.5, 1.0, -1.0, float("nan"), float("inf")):
        assert append(lib, rope=rope) == BAD
    assert append(lib, givens=3) == BAD and append(lib, pages(H=3)) == BAD and append(lib, pages(H=3), givens=0) == HIP
    assert append(lib, theta=None) == BAD and append(lib, theta=None, givens=0) == HIP
    assert append(lib, q=None, qo=None) == HIP and append(lib, qo=None) == BAD
    assert append(lib, s=(-1, 64, 128, 64)) == BAD and append(lib, s=(128, 64, 1 << 40, 64)) == UNSUP
    for n in ("k", "v", "slots", "positions", "kc", "vc"):
        assert append(lib, **{n: None}) == BAD
        assert append(lib, **{n: A[12] + 1}) == BAD
    assert append(lib, kc=A[12] + 8) == BAD and append(lib, qo=A[12] + 8) == BAD
    assert append(lib, k=A[12] + 2) == HIP  # rows on any element
    # overlaps: the pools with each other, with inputs, with q_out
    assert append(lib, vc=A[7]) == BAD and append(lib, kc=A[0]) == BAD and append(lib, qo=A[7] + 64) == BAD
    assert append(lib, qo=A[1]) == BAD and append(lib, vc=A[7] + 32 * 64 * 2) == BAD
    # one allocation [pages, 2, H, page, D] holds both
    joint = pages(sp=2 * 2 * 16 * 64)
    assert append(lib, joint, vc=A[7] + 2 * 16 * 64 * 2) == HIP and append(lib, joint, vc=A[7] + 16 * 64 * 2) == BAD


# ---------------------------------------------------------------------------
def decode(lib, c=None, B=3, Hq=4, W=40, top=0, tau=2.0, scale=0.0, ws_bytes=1 << 23, **kw):
    a = {n: A[i] for i, n in enumerate("q kc vc table lengths lam out stat ws".split())}
    a.update(kw)
    c = pages(P=100) if c is None else c
    d = R.RelPagedQuery(B, Hq, W, top, tau, scale)
    return lib.relation_paged_decode(ctypes.byref(c), ctypes.byref(d), a["q"], a["kc"], a["vc"], a["table"], a["lengths"],
                                     a["lam"], a["out"], a["stat"], a["ws"], ws_bytes, None)


@pytest.mark.parametrize("c,code", POOLS)
def test_decode_pool(lib, c, code):
    assert decode(lib, pages(**c)) == code


def test_decode_arguments(lib):
    nan = float("nan")
    assert decode(lib, B=0) == OK and decode(lib, Hq=0) == OK and decode(lib, B=-1) == BAD
    assert decode(lib, Hq=5) == BAD and decode(lib, W=0) == BAD and decode(lib, W=1 << 27) == UNSUP
    assert decode(lib, tau=0.0) == BAD and decode(lib, tau=nan) == BAD and decode(lib, scale=nan) == BAD
    assert decode(lib, B=1 << 20, Hq=1 << 12) == UNSUP
    for n in ("q", "kc", "vc", "table", "lengths", "lam", "out"):
        assert decode(lib, **{n: None}) == BAD
        assert decode(lib, **{n: A[12] + 2}) == BAD
    assert decode(lib, stat=None) == HIP and decode(lib, q=A[12] + 8) == BAD and decode(lib, W=400, ws=A[12] + 8) == BAD
    for n in ("q", "kc", "vc", "table", "lengths", "lam"):
        assert decode(lib, out=A["q kc vc table lengths lam".split().index(n)]) == BAD
    assert decode(lib, stat=A[6]) == BAD and decode(lib, W=400, ws=A[1]) == BAD


def test_decode_workspace(lib):
    c = pages(P=100)
    need = lambda W, top, B=3: lib.relation_paged_decode_workspace_bytes(
        ctypes.byref(c), ctypes.byref(R.RelPagedQuery(B, 4, W, top, 2.0, 0.0)))
    big = need(4000, 0)
    assert big >= 2 * 12 * 66 * 4 and need(4000, 0, B=0) == 0
    assert need(4000, 20) == 0                      # one slice a row: nothing to join
    assert decode(lib, W=4000, ws_bytes=big) == HIP and decode(lib, W=4000, ws_bytes=big - 1) == WS
    assert decode(lib, W=4000, ws=None, ws_bytes=big) == WS
    assert decode(lib, W=4000, top=20, ws=None, ws_bytes=0) == HIP
    assert lib.relation_paged_decode_workspace_bytes(None, None) == 0


# ---------------------------------------------------------------------------
def sample(lib, B=3, V=1000, dtype=R.REL_BF16, sl=None, sn=None, ws_bytes=1 << 23, **kw):
    a = {n: A[i] for i, n in enumerate("x r T k p mp tokens lp ws".split())}
    a.update(kw)
    s = R.RelSample(B, V, dtype, V if sl is None else sl, V if sn is None else sn)
    return lib.relation_sample(ctypes.byref(s), a["x"], a["r"], a["T"], a["k"], a["p"], a["mp"], a["tokens"], a["lp"],
                               a["ws"], ws_bytes, None)


def test_sample_arguments(lib):
    assert sample(lib) == HIP and sample(lib, B=0) == OK and sample(lib, B=-1) == BAD and sample(lib, V=0) == BAD
    assert sample(lib, V=(1 << 22) + 1) == UNSUP and sample(lib, B=(1 << 20) + 1) == UNSUP and sample(lib, dtype=2) == UNSUP
    assert sample(lib, sl=999) == BAD and sample(lib, sn=999) == BAD and sample(lib, B=1, sl=0, sn=0) == HIP
    assert sample(lib, sl=1 << 50) == UNSUP
    for n in ("x", "r", "tokens"):
        assert sample(lib, **{n: None}) == BAD
    assert sample(lib, T=None, k=None, p=None, mp=None, lp=None) == HIP
    for n in ("r", "T", "k", "p", "mp", "lp", "tokens"):
        assert sample(lib, **{n: A[12] + 2}) == BAD
    assert sample(lib, x=A[12] + 2) == HIP and sample(lib, x=A[12] + 1) == BAD
    for n in range(6):
        assert sample(lib, tokens=A[n]) == BAD
    assert sample(lib, lp=A[6]) == BAD
    s = R.RelSample(3, 100000, R.REL_F32, 100000, 100000)
    need = lib.relation_sample_workspace_bytes(ctypes.byref(s))
    if need:
        assert sample(lib, V=100000, dtype=R.REL_F32, ws_bytes=need - 1) == WS
        assert sample(lib, V=100000, dtype=R.REL_F32, ws=None, ws_bytes=need) == WS
    assert sample(lib, V=100000, dtype=R.REL_F32, ws_bytes=need) == HIP
    assert lib.relation_sample_workspace_bytes(None) == 0


def test_injected_launch_failure(lib, monkeypatch):
    monkeypatch.setenv("RELATION_TEST_FAIL_LAUNCH", "1")
    for call in (page_map, append, decode, sample):
        assert call(lib) == HIP and b"injected" in lib.relation_last_error()


def test_sample_row_strides(lib):
    """0 is one row for all; rows are only read."""
    assert sample(lib, sl=0) == HIP and sample(lib, sn=0) == HIP and sample(lib, sl=0, sn=0) == HIP
    for bad in (-1000, -1, 1, 999):
        assert sample(lib, sl=bad) == BAD and sample(lib, sn=bad) == BAD


def test_accepted_calls_end_before_the_launch(lib):
    """What every other test here relies on, for each entry point."""
    for call in (page_map, append, decode, sample):
        assert call(lib) == HIP and b"injected" in lib.relation_last_error(), call.__name__


def test_overlaps_are_named(lib):
    for call, out, other in ((page_map, "counts", 0), (append, "qo", 1), (decode, "stat", 6), (sample, "lp", 6)):
        assert call(lib, **{out: A[other]}) == BAD and b"overlaps" in lib.relation_last_error(), call.__name__


def test_long_rows_need_a_workspace(lib):
    """Rows over 8192 fp32 or 16384 bf16 logits take two kernels and a workspace between them."""
    need = lambda V, dt: lib.relation_sample_workspace_bytes(ctypes.byref(R.RelSample(3, V, dt, V, V)))
    for dt, most in ((R.REL_F32, 8192), (R.REL_BF16, 16384)):
        assert need(most, dt) == 0 and need(most + 1, dt) > 0 and need(100000, dt) > 0


def test_whole_numbers_past_32_bits():
    """They become the nearest number that fits, or no position; not the low half of their bits."""
    far, top = 1 << 32, 2 ** 31 - 1
    x = torch.tensor([far + 5, -far + 5, 7, top + 1, -1, 0])
    assert R._int32(x).tolist() == [top, -top - 1, 7, top, -1, 0] and R._int32(x).dtype == torch.int32
    assert R._positions(x).tolist() == [-1, -top - 1, 7, -1, -1, 0]
    assert R._int32(torch.tensor([3e9, 5.0, float("nan"), float("inf")])).tolist() == [top, 5, -1, top]
    assert R._int32(torch.tensor([200, 3], dtype=torch.uint8)).tolist() == [200, 3]
    assert R._positions(torch.tensor([top], dtype=torch.int32)).tolist() == [top]
    y = torch.arange(6, dtype=torch.int32)
    assert R._int32(y) is y and R._int32(y[::2]).tolist() == [0, 2, 4] and R._int32(x.view(2, 3).t()).is_contiguous()
    _, k = R._per_row(1 << 40, "top_k", 2, torch.int32, torch.zeros(2, 3))
    assert k.tolist() == [top, top]


def test_binding_refuses_what_is_not_on_the_gpu(lib):
    x = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        R.relation_page_map(x, x, x.view(3, 1), x, 16, 3)
    with pytest.raises(ValueError, match="on the GPU"):
        R.relation_sample(torch.zeros(2, 8), torch.ones(2, 8))
    kc = torch.zeros(4, 2, 16, 64)
    with pytest.raises(ValueError, match="on the GPU"):
        R.relation_paged_decode(torch.zeros(3, 2, 64), kc, kc, x.view(3, 1), x, 0.5)
    with pytest.raises(ValueError, match="share shape"):
        R.make_pages(kc, kc.transpose(1, 2))
    with pytest.raises(ValueError, match="contiguous"):
        R.make_pages(kc.transpose(2, 3), kc.transpose(2, 3))
