"""A fork whose copy takes page 0 while other rows have nothing to copy: these leave page 0 alone, whose number is what a sum over no open page, or an
entry that nobody set, would be."""
import pytest
import torch

from gpu_util import announce
from test_kv_pages_gpu import Book, cache_of, dev, moved

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pages", [9, 16385])
@pytest.mark.parametrize("parents", [[0, 1, 0, 2, 1, 3], [1, 1, 3, 0, 0], [2, 0, 0, -1, 9, 1]])
def test_page_zero_is_taken(pages, parents):
    announce("fork, page 0", pages, parents)
    # an open page; full pages alone; nothing; an open page that is no page
    rows = [([3, 4], 40), ([1, 2], 64), ([], 0), ([5, -1], 50)]
    c, book = cache_of(pages, seed=3), Book(pages, 32, 3, rows)
    before, args = c.data.clone(), (dev(book.table()), dev(book.lengths), dev(book.uses))
    book.fork(parents)
    assert book.copies == [(4, 0)]
    for _ in range(3):                                              # (the source of the copy stays: each run gives the same)
        got = c.fork(*args, dev(parents))
        assert got[0].tolist() == book.table() and got[1].tolist() == book.lengths and got[2].tolist() == book.uses
        assert torch.equal(c.data, moved(before, book.copies)) and not torch.equal(before[0], before[4])
