"""Pages given out to documents by the host (no GPU work)."""
import pytest
import torch

from paper_2401_06145_amd import transformer as tr


def caches(docs=3, pages=8, page=4, most=5):
    model = tr.Transformer(tr.Config(width=32, heads=2, kv_heads=1, layers=1, inner=32), device="cpu")
    return model.pages(docs, pages, page=page, most=most)


def test_pages_are_given_out_and_back():
    c = caches()
    c.grow([5, 0, 1])
    assert c.lens == [5, 0, 1] and c.length.tolist() == [5, 0, 1]
    assert [len(h) for h in c.held] == [2, 0, 1] and len(c.free) == 5
    c.grow([3, 1, 0])  # the first document's second page has room
    assert [len(h) for h in c.held] == [2, 1, 1] and len(c.free) == 4
    for t, held in enumerate(c.held):
        assert c.table[t, :len(held)].tolist() == held
    every = sum(c.held, []) + c.free
    assert sorted(every) == list(range(8))
    c.release(0)
    assert c.lens == [0, 1, 1] and c.length.tolist() == [0, 1, 1] and len(c.free) == 6
    c.grow([20, 0, 0])
    assert len(c.held[0]) == 5 and sorted(sum(c.held, []) + c.free) == list(range(8))


@pytest.mark.parametrize("new", [[21, 0, 0], [20, 20, 0], [1, 1], [1, -1, 0]])
def test_what_does_not_fit_changes_nothing(new):
    c = caches()
    c.grow([1, 2, 3])
    with pytest.raises(ValueError):
        c.grow(new)
    assert c.lens == [1, 2, 3] and [len(h) for h in c.held] == [1, 1, 1] and len(c.free) == 5


def test_heads_that_do_not_turn_ask_for_nothing():
    model = tr.Transformer(tr.Config(width=32, heads=2, kv_heads=1, layers=1, inner=32), device="cpu")
    assert model._places(3, torch.tensor([0, 3])) is None and len(model.freq) == 0
    assert "g_q" not in model.layers[0]
    turned = tr.Transformer(tr.Config(width=32, heads=2, kv_heads=1, layers=1, inner=32, rotary=8, head_norm=True), device="cpu")
    start, first = torch.tensor([0, 2, 2, 5], dtype=torch.int32), torch.tensor([7, 9, 0], dtype=torch.int32)
    assert turned._places(5, start, first).tolist() == [7, 8, 0, 1, 2]
    # and the weights that were there before are the same
    assert torch.equal(model.layers[0]["g_down"], turned.layers[0]["g_down"])


def state(c):
    return (list(c.lens), c.length.tolist(), [list(h) for h in c.held], list(c.free),
            [c.table[t, :len(h)].tolist() for t, h in enumerate(c.held)])


@pytest.mark.parametrize("rows,new", [
    (torch.zeros((6, 31)), [5, 0, 1]), (torch.zeros((6, 32, 1)), [5, 0, 1]), (torch.zeros((6, 32), dtype=torch.float64), [5, 0, 1]),
    (torch.zeros((6, 32), device="meta"), [5, 0, 1]),
    (torch.zeros((6, 32)), [5, 0, 1]),  # rows as they should be, which the operators refuse: they are not on a GPU
    (torch.zeros((6, 32), requires_grad=True), [5, 0, 1]), (torch.zeros((5, 32)), [5, 0, 1]), (torch.zeros((21, 32)), [21, 0, 0]),
])
def test_a_refused_call_leaves_the_caches_as_they_were(rows, new):
    model = tr.Transformer(tr.Config(width=32, heads=2, kv_heads=1, layers=1, inner=32), torch.float32, device="cpu")
    c = model.pages(3, 8, page=4, most=5)
    c.grow([3, 9, 0])
    c.release(0)
    c.grow([2, 0, 1])
    before = state(c)
    with pytest.raises((ValueError, TypeError, RuntimeError)):
        model.extend(rows, new, c)
    assert state(c) == before
    # and what comes next gets the pages that it would have got
    c.grow([5, 0, 1])
    d = model.pages(3, 8, page=4, most=5)
    d.grow([3, 9, 0])
    d.release(0)
    d.grow([2, 0, 1])
    d.grow([5, 0, 1])
    assert state(c) == state(d)


@pytest.mark.parametrize("page", [0, -4, 3, 48, 1 << 17])
def test_pages_that_no_call_takes(page):
    with pytest.raises(ValueError):
        caches(page=page)


def test_tokens_taken_back():
    c = caches()
    c.grow([5, 0, 1])
    before = state(c)
    c.grow([6, 4, 0])
    c.shrink([6, 4, 0])
    assert state(c) == before
    c.grow([0, 0, 0])
    c.shrink([0, 0, 0])
    assert state(c) == before
