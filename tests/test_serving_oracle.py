"""Pins of the serving oracle: closed forms and other routes than the ones it takes."""
from __future__ import annotations

import math

import numpy as np
import pytest

from oracle import decode_oracle as DO
from oracle import layer_oracle as LO
from oracle import serving_oracle as SO


def test_page_map_by_hand():
    table = np.full((4, 3), -1)
    table[0, :2] = [7, 8]
    table[2, 0] = 3
    m = SO.page_map([6, 0, 4, 0], [1, 5, 1, 0], table, [20, 21, 22, 23], 4, 9)
    # 6 + 1 tokens stay in two pages; 5 tokens take two; 4 + 1 take a second; nothing for the last
    assert m["table"].tolist() == [[7, 8, -1], [20, 21, -1], [3, 22, -1], [-1, -1, -1]]
    assert m["lengths"].tolist() == [7, 5, 5, 0] and m["row_start"].tolist() == [0, 1, 6, 7, 7]
    assert m["slots"].tolist() == [8 * 4 + 2, 80, 81, 82, 83, 84, 88, -1, -1]
    assert m["positions"].tolist() == [6, 0, 1, 2, 3, 4, 4, -1, -1] and m["counts"].tolist() == [3, 7, 0]


def test_page_map_refusals_by_hand():
    table = np.full((5, 2), -1)
    # -1 cached; a row of two pages cannot hold 9 tokens; two pages needed where one is left; one with nothing to add
    m = SO.page_map([-1, 0, 0, 0, 4], [1, 9, 3, 8, 0], table, [5, 6], 4, 100)
    assert m["lengths"].tolist() == [0, 0, 3, 0, 4] and m["counts"].tolist() == [1, 3, 3]
    assert m["table"].tolist() == [[-1, -1], [-1, -1], [5, -1], [-1, -1], [-1, -1]]
    assert (m["slots"] >= 0).sum() == 3 and m["slots"][10:13].tolist() == [20, 21, 22]
    # a step's buffers that end inside a request's tokens
    m = SO.page_map([0, 0], [3, 3], np.full((2, 2), -1), [1, 2], 4, 5)
    assert m["lengths"].tolist() == [3, 0] and m["row_start"].tolist() == [0, 3, 5] and m["counts"].tolist() == [1, 3, 1]


def test_turned_is_the_layers_rope():
    x = np.random.default_rng(3).standard_normal((2, 9, 12))
    want = LO.rope(x, 1.0e4)
    for t in range(9):
        assert np.allclose(SO.turned(x[:, t], t, 1.0e4), want[:, t], atol=1e-12)


def test_append_puts_rows_where_the_slots_say():
    rng = np.random.default_rng(4)
    k, v, q = (rng.standard_normal((3, 2, 4)) for _ in range(3))
    kc, vc = rng.standard_normal((2, 2, 4, 6)), rng.standard_normal((2, 2, 4, 6))
    nk, nv, nq = SO.append(k, v, kc, vc, [5, -1, 8], [0, 1, 0], q=q)  # the second and third are outside the pool
    assert np.array_equal(nk[1, :, 1, :4], k[0]) and not nk[1, :, 1, 4:].any() and np.array_equal(nv[1, :, 1, :4], v[0])
    nk[1, :, 1], nv[1, :, 1] = kc[1, :, 1], vc[1, :, 1]
    assert np.array_equal(nk, kc) and np.array_equal(nv, vc) and not nq[1:].any()


def test_paged_decode_is_decode_of_the_gathered_cache():
    rng = np.random.default_rng(5)
    P, H, page, D = 9, 2, 4, 8
    kc, vc = rng.standard_normal((P, H, page, D)), rng.standard_normal((P, H, page, D))
    table = [[4, 0, 8], [2, 7, -1]]
    q = rng.standard_normal((2, 4, D))
    Y, M = SO.paged_decode(q, kc, vc, table, [10, 8], 0.3)
    k = np.concatenate([kc[4, 1], kc[0, 1], kc[8, 1]])
    v = np.concatenate([vc[4, 1], vc[0, 1], vc[8, 1]])
    y, m = DO.decode_step(q[0, 2], k, v, 10, 0.3)
    assert np.allclose(Y[0, 2], y) and abs(M[0, 2] - m) < 1e-12
    Y, _ = SO.paged_decode(q, kc, vc, table, [13, 9], 0.3)  # past the table; a page of -1
    assert np.isnan(Y).all()


def test_sample_by_hand_and_by_frequency():
    x = np.log([0.5, 0.2, 0.2, 0.1])
    one = np.ones(4)
    pick = lambda **kw: SO.sample(x, one, **kw)["kept"]
    assert pick() == [0, 1, 2, 3] and pick(top_k=2) == [0, 1] and pick(temperature=0) == [0]
    assert pick(top_p=0.6) == [0, 1] and pick(top_p=0.71) == [0, 1, 2] and pick(top_p=0.0) == [0]
    assert pick(min_p=0.3) == [0, 1, 2] and pick(min_p=0.5) == [0] and pick(min_p=2.0) == [0]
    assert abs(SO.sample(x, one, temperature=0.5)["logprob"] - math.log(0.25 / 0.34)) < 1e-12
    rng = np.random.default_rng(6)
    n = 20000
    hits = np.bincount([SO.sample(x, rng.exponential(size=4), top_p=0.71)["token"] for _ in range(n)], minlength=4)
    want = np.array([5, 2, 2, 0]) / 9
    assert hits[3] == 0 and np.all(np.abs(hits / n - want) < 5 * np.sqrt(want * (1 - want) / n) + 1e-9)


@pytest.mark.parametrize("row", [[-math.inf] * 3, [math.nan] * 3])
def test_sample_of_nothing(row):
    assert SO.sample(row, np.ones(3))["token"] == -1


def test_sample_masks_and_infinities():
    low = -3.4028234663852886e38
    assert SO.sample([low, 0.0, -math.inf, math.nan], np.ones(4), top_k=3)["kept"][:2] == [1, 0]
    assert SO.sample([math.inf, 1.0, math.inf], np.array([2.0, 0.1, 1.0]))["token"] == 2
    assert SO.sample([low, low], np.array([2.0, 1.0]))["token"] == 1  # a row of the type's lowest value is even
