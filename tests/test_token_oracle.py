"""Pins of the oracle of the norms with rotation and of the log-probabilities: closed forms worked by hand, other
routes, central differences."""
from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import layer_oracle, serving_oracle
from oracle import token_oracle as TO

RNG = np.random.default_rng(3)


def test_norm_of_known_rows():
    x = np.array([3.0, 4.0, 0.0, 0.0]).reshape(1, 1, 1, 4)
    zero = np.zeros((1, 1), int)
    y = TO.norm_rope(x, None, zero, eps=1e-12)  # mean square 25/4
    assert np.allclose(y.ravel(), [1.2, 1.6, 0, 0], atol=1e-11)
    y = TO.norm_rope(x, [1, 2, 3, 4], zero, eps=6.25 * 3)  # sqrt(6.25 * 4) = 5
    assert np.allclose(y.ravel(), [0.6, 1.6, 0, 0], atol=1e-12)
    assert not TO.norm_rope(np.zeros((1, 1, 1, 4)), None, zero).any()


@pytest.mark.parametrize("layout,a,b", [("half", 0, 2), ("half", 1, 3), ("interleaved", 0, 1), ("interleaved", 2, 3)])
def test_pairs_turn_together(layout, a, b):
    """A quarter turn of a pair; base 100 turns the second pair by a tenth of the first's angle."""
    w = TO.frequencies(4, 100.0)
    assert np.allclose(w, [1.0, 0.1])
    R = TO.rotation(6, 4, 3, layout, base=100.0)
    ang = 3.0 * (1.0 if (a, b) in ((0, 2), (0, 1)) else 0.1)
    assert math.isclose(R[a, a], math.cos(ang)) and math.isclose(R[b, a], math.sin(ang)) and math.isclose(R[a, b], -math.sin(ang))
    assert R[4, 4] == R[5, 5] == 1.0 and not R[4, :4].any()


def test_half_layout_is_the_layer_oracles_rotation():
    x = RNG.standard_normal((1, 2, 7, 16))
    pos = np.arange(7)[None] * 13
    y = TO.norm_rope(x, None, pos, norm=False)
    for t in range(7):
        assert np.allclose(y[0, :, t], serving_oracle.turned(x[0, :, t], 13 * t, 1.0e4))
    assert np.allclose(TO.norm_rope(x, None, np.arange(7)[None], norm=False), layer_oracle.rope(x))


def test_interleaved_is_half_with_the_channels_in_another_order():
    x = RNG.standard_normal((1, 1, 3, 12))
    pos = np.array([[0, 5, 900]])
    order = [0, 4, 1, 5, 2, 6, 3, 7, 8, 9, 10, 11]  # place of half's channel in the interleaved row
    h = TO.norm_rope(x, None, pos, rope_dim=8)
    z = np.empty_like(x)
    z[..., :] = x[..., order]
    i = TO.norm_rope(z, None, pos, rope_dim=8, layout="interleaved")
    assert np.allclose(i, h[..., order])


def test_scaled_frequencies():
    """Slow pairs are divided by the factor, fast ones kept, those between mixed; without a length all are divided."""
    base = TO.frequencies(64)
    w = TO.frequencies(64, factor=8.0, original_length=2048)
    often = [2048 * b / (2 * math.pi) for b in base]
    for b, x, o in zip(base, w, often):
        if o >= 32:
            assert x == b
        elif o <= 1:
            assert math.isclose(x, b / 8)
        else:
            assert b / 8 < x < b
    assert any(o >= 32 for o in often) and any(o <= 1 for o in often) and any(1 < o < 32 for o in often)
    assert np.allclose(TO.frequencies(64, factor=8.0), np.array(base) / 8)
    mid = TO.frequencies(2, factor=3.0, original_length=100, low=100 / (2 * math.pi) - 1, high=100 / (2 * math.pi) + 3)[0]
    assert math.isclose(mid, 0.25 + 0.75 / 3)  # a quarter of the way up


@pytest.mark.parametrize("kw", [dict(), dict(layout="interleaved", rope_dim=4), dict(norm=False, rope_dim=6),
                                dict(factor=4.0, original_length=64, amplitude=1.3), dict(rope_dim=0)])
def test_norm_gradients_by_differences(kw):
    x, w, dy = RNG.standard_normal((2, 2, 3, 8)), 1 + 0.3 * RNG.standard_normal(8), RNG.standard_normal((2, 2, 3, 8))
    pos = np.array([[0, 7, 1000], [3, -1, 2]])
    w = w if kw.get("norm", True) else None
    dx, dw = TO.norm_rope_backward(x, w, pos, dy, **kw)
    f = lambda x, w: float(np.sum(dy * TO.norm_rope(x, w, pos, **kw)))
    e = 1e-6
    for _ in range(20):
        i = tuple(RNG.integers(0, n) for n in x.shape)
        d = np.zeros_like(x)
        d[i] = e
        assert abs((f(x + d, w) - f(x - d, w)) / (2 * e) - dx[i]) < 1e-7 * (1 + abs(dx[i]))
    if w is not None:
        for i in range(8):
            d = np.zeros(8)
            d[i] = e
            assert abs((f(x, w + d) - f(x, w - d)) / (2 * e) - dw[i]) < 1e-7 * (1 + abs(dw[i]))
    assert not dx[1, :, 1].any()


def test_logprobs_of_known_rows():
    r = TO.logprobs([0.0, math.log(3.0)], 0, 2)  # p = 1/4, 3/4
    assert math.isclose(r["logprob"], math.log(0.25)) and r["rank"] == 1 and r["top_tokens"] == [1, 0]
    assert math.isclose(r["entropy"], -0.25 * math.log(0.25) - 0.75 * math.log(0.75))
    r = TO.logprobs([2.0] * 8, 5, 3)
    assert math.isclose(r["entropy"], math.log(8)) and r["rank"] == 5 and r["top_tokens"] == [0, 1, 2]
    r = TO.logprobs([math.inf, 0.0, math.inf, math.nan, -math.inf], 1, 5)
    assert r["logprob"] == -math.inf and math.isclose(r["entropy"], math.log(2)) and r["top_tokens"] == [0, 2, 1, 3, 4]
    assert TO.logprobs([1.0, 2.0], -1)["logprob"] == 0.0 and math.isnan(TO.logprobs([1.0, 2.0], 2)["logprob"])
    assert math.isnan(TO.logprobs([-math.inf, math.nan], 0)["entropy"])
    assert TO.logprobs([-math.inf, math.nan], -1)["logprob"] == 0.0
    assert not TO.logprobs_backward([-math.inf, math.nan], -1, 2.0, 0.0).any()


def test_logprob_gradients_by_differences():
    x = RNG.standard_normal(9) * 2
    for token in (0, 4, -3):
        d = TO.logprobs_backward(x, token, 0.7, -1.3)

        def f(x):
            r = TO.logprobs(x, token)
            return 0.7 * r["logprob"] - 1.3 * r["entropy"]
        for i in range(9):
            e = np.zeros(9)
            e[i] = 1e-6
            assert abs((f(x + e) - f(x - e)) / 2e-6 - d[i]) < 1e-8
        assert abs(d.sum()) < 1e-14


def test_chunks_are_decode_steps():
    """Every row of a chunk is the decode step at its position; a bad page spoils the rows from it on."""
    H, G, D, page = 2, 2, 8, 4
    kc, vc = RNG.standard_normal((2, 6, H, page, D))
    q = RNG.standard_normal((7, H * G, D))
    table, lens, start = [[4, 0, 2], [5, 9, 0]], [9, 6], [0, 4, 7]
    Y, M = serving_oracle.paged_prefill(q, kc, vc, table, lens, start, 0.3)
    for r, n in enumerate((6, 7, 8, 9)):
        y, m = serving_oracle.paged_decode(q[r][None], kc, vc, [table[0]], [n], 0.3)
        assert np.array_equal(Y[r], y[0]) and np.array_equal(M[r], m[0])
    assert not np.isnan(Y[4]).any() and np.isnan(Y[5]).all() and np.isnan(Y[6]).all()
    Y, _ = serving_oracle.paged_prefill(q, kc, vc, table, [3, 14], start, 0.3)
    assert all(np.isnan(y).all() for y in Y)
