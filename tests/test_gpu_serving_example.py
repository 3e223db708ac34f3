"""The serving example end to end: prompts and decode steps through the paged
cache give the hidden rows that the whole sequences give, and the same tokens
whatever the page size."""
from __future__ import annotations

import pytest
import torch

from examples import serve_paged as E

pytestmark = pytest.mark.gpu

# Both paths round the rotated operands, the outputs and the residual to bf16 in each of two layers, in other
# places: relative 2^-8 a rounding, eight of them, at their square root and doubled.
BAR = 2.0 ** -8 * 8 ** 0.5 * 2


@pytest.fixture(scope="module")
def model():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return E.Decoder(vocab=3001, layers=2, heads=4, width=64)


def _prompts(model, lens):
    g = torch.Generator(device="cuda").manual_seed(7)
    return [torch.randint(0, model.emb.shape[0], (n,), device="cuda", generator=g) for n in lens]


@pytest.mark.parametrize("page", [8, 32])
def test_decode_steps_are_the_whole_sequence(model, page):
    prompts = _prompts(model, (1, 15, 33, 290))
    tokens, logprob, x = E.generate(model, prompts, 20, page_size=page, temperature=0.8, top_k=50, top_p=0.9)
    torch.cuda.synchronize()
    err = E.check(model, prompts, tokens, x)
    print(f"page {page}: relative 2-norm {err:.2e} (bar {BAR:.2e})", flush=True)
    assert err <= BAR
    assert tokens.shape == (4, 20) and int(tokens.min()) >= 0 and int(tokens.max()) < 3001
    assert bool((logprob <= 0).all())


def test_page_size_changes_nothing(model):
    prompts = _prompts(model, (5, 64))
    a, b = (E.generate(model, prompts, 12, page_size=p, temperature=0.0)[0] for p in (16, 64))
    assert torch.equal(a, b)


@pytest.mark.parametrize("width", [60, 36])
def test_heads_narrower_than_the_cache(width):
    """Heads that the caches pad: the decode steps keep the scale of the true width."""
    narrow = E.Decoder(vocab=3001, layers=2, heads=4, width=width)
    prompts = _prompts(narrow, (1, 40, 200))
    tokens, _, x = E.generate(narrow, prompts, 12, page_size=16, temperature=0.8, top_k=50)
    torch.cuda.synchronize()
    err = E.check(narrow, prompts, tokens, x)
    print(f"width {width}: relative 2-norm {err:.2e} (bar {BAR:.2e})", flush=True)
    assert err <= BAR


def test_a_step_that_does_not_fit_changes_nothing(model):
    """The requests keep their places, and a smaller step goes on from them."""
    pool = E.Pool(model, 2, 3, 16, 40)
    pool.step([16, 15])
    for added in ([17, 2], [0, 40]):  # two pages of the one left; a longer row than the table's
        with pytest.raises(RuntimeError, match="pages needed"):
            pool.step(added)
        assert pool.lengths.tolist() == [16, 15] and pool.count == [16, 15] and pool.taken == 2
    m = pool.step([3, 1])
    assert m["lengths"].tolist() == [19, 16] and m["positions"].tolist() == [16, 17, 18, 15] and m["counts"].tolist() == [1, 4, 0]


def test_a_request_that_waits_for_a_page_goes_on_from_its_place(model):
    """The map alone, with the lengths of unserved requests kept as its documentation says."""
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    table, lengths = i32([[0, -1], [1, -1]]), i32([16, 16])
    m = E.R.relation_page_map(lengths, i32([1, 1]), table, i32([2]), 16, 2)
    assert m["lengths"].tolist() == [17, 0] and m["counts"].tolist() == [1, 1, 1]
    lengths = torch.where(m["lengths"] > 0, m["lengths"], lengths)
    m = E.R.relation_page_map(lengths, i32([1, 1]), table, i32([3]), 16, 2)
    assert m["lengths"].tolist() == [18, 17] and m["positions"].tolist() == [17, 16]
    assert m["slots"].tolist() == [2 * 16 + 1, 3 * 16] and table.tolist() == [[0, 2], [1, 3]]
