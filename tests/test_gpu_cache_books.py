"""Books of the cache where tables have gaps: no page is lost, whatever was refused, committed, evicted or rolled back."""
from __future__ import annotations

import numpy as np
import pytest

from tests import cache_reference as R
from tests.test_gpu_cache_pages import _i32, _pair, _same
import paper_2512_18337_b200 as S

pytestmark = pytest.mark.gpu
DROP = -(1 << 31)


class Books(R.Books):
    """A commit gives up every page behind the new length, gaps or not."""

    def commit(self, rows):
        gone = []
        for s, n in rows:
            if not 0 <= s < len(self.len):
                continue
            self.len[s] = min(max(int(self.len[s]) + n, 0), self.max_pages * self.P)
            for i in range(self.held(s), self.max_pages):
                if self.table[s, i] >= 0:
                    gone.append(int(self.table[s, i]))
                    self.table[s, i] = -1
        for p in gone:
            self.ref[p] -= 1
        for p in dict.fromkeys(gone):
            if self.ref[p] == 0:
                self.free.append(p)


def _books(n_pages, P, n_streams, max_pages, seed=0):
    c, plain, rng = _pair(n_pages, P, n_streams, max_pages, seed=seed)
    return c, Books(n_pages, P, n_streams, max_pages, plain.pages), rng


def _whole(c):
    """Counts equal the holders, and every page is held or on the free list, once."""
    table = c.page_table.cpu().numpy()
    ref = c.ref_count.cpu().numpy()
    held = table[table >= 0]
    assert (np.bincount(held, minlength=len(ref)) == ref).all()
    free = c.free_list[:c.status()[0]].tolist()
    assert sorted(free) == np.flatnonzero(ref == 0).tolist()


def _both(c, book, call, rows):
    getattr(c, call)(_i32([n for _, n in rows]), streams=_i32([s for s, _ in rows]))
    getattr(book, call)(rows)
    _same(c, book)
    _whole(c)


def test_a_refused_reserve_and_what_follows():
    """2,048 tokens are refused and committed all the same; the next reserve stands behind the gap; then the stream is dropped."""
    c, book, _ = _books(20, 16, 3, 200)
    _both(c, book, "reserve", [(0, 20), (1, 5)])
    _both(c, book, "commit", [(0, 20), (1, 5)])
    _both(c, book, "reserve", [(0, 2048)])
    assert c.status()[1] == S.SAM_CACHE_OUT_OF_PAGES
    _both(c, book, "commit", [(0, 2048)])
    _both(c, book, "reserve", [(0, 40)])
    assert int(c.page_table[0, 129]) >= 0 and int(c.page_table[0, 128]) == -1
    _both(c, book, "commit", [(0, 3)])
    _both(c, book, "commit", [(0, -1000)])                 # into the gap
    assert int((c.ref_count > 0).sum()) == 3
    _both(c, book, "reserve", [(0, 100)])
    _both(c, book, "commit", [(0, DROP)])
    assert (c.page_table[0] == -1).all() and int((c.ref_count > 0).sum()) == 1


def test_evicted_pages_do_not_hide_the_others():
    """The caller took the oldest pages, and one in the middle, out of the table; rolling back and dropping find the rest."""
    c, book, _ = _books(100, 32, 3, 60, seed=1)
    _both(c, book, "reserve", [(0, 900), (1, 700)])
    _both(c, book, "commit", [(0, 850), (1, 700)])
    for s, i in ((0, 0), (0, 1), (0, 2), (0, 15), (1, 0)):
        page = int(c.page_table[s, i])
        n_free = int(c.meta[0])
        c.page_table[s, i], c.ref_count[page], c.free_list[n_free], c.meta[0] = -1, 0, page, n_free + 1
        book.table[s, i], book.ref[page] = -1, 0
        book.free.append(page)
    _same(c, book)
    _whole(c)
    c.fork(_i32([0]), _i32([2]))
    book.fork([(0, 2)])
    _same(c, book)
    _both(c, book, "reserve", [(2, 3), (0, 3)])
    _both(c, book, "commit", [(0, -400), (2, 1)])
    _both(c, book, "commit", [(1, DROP), (0, DROP)])
    _both(c, book, "commit", [(2, DROP)])
    assert c.status()[0] == 100


@pytest.mark.parametrize("max_pages,at", [(3, 1), (3, 2), (700, 256), (700, 699)])
def test_fork_refuses_a_row_with_a_page_anywhere(max_pages, at):
    """No tokens and no first page, but a page further on (the caller's table): it would be lost."""
    c, book, _ = _books(12, 16, 3, max_pages, seed=2)
    _both(c, book, "reserve", [(0, 20)])
    _both(c, book, "commit", [(0, 20)])
    page, n_free = book.free.pop(), int(c.meta[0])
    c.page_table[1, at], c.ref_count[page], c.meta[0] = page, 1, n_free - 1
    book.table[1, at], book.ref[page] = page, 1
    c.fork(_i32([0, 0]), _i32([1, 2]))
    book.fork([(0, 2)])
    book.status = S.SAM_CACHE_BAD_FORK
    _same(c, book)
    _whole(c)


@pytest.mark.parametrize("P,n_streams,max_pages,n_pages", [(16, 5, 9, 24), (32, 40, 6, 120), (16, 33, 90, 700), (64, 1100, 5, 2500), (16, 3, 700, 900)])
def test_random_walk_with_gaps(P, n_streams, max_pages, n_pages):
    """Commits by any number of tokens, whatever was reserved before them, or refused."""
    c, book, rng = _books(n_pages, P, n_streams, max_pages, seed=P + n_streams)
    for step in range(60):
        what = rng.choice(["reserve", "reserve", "commit", "commit", "back", "drop", "fork", "compact"])
        some = rng.permutation(n_streams)[:rng.integers(1, n_streams + 1)].tolist()
        if what in ("reserve", "commit", "back", "drop"):
            lo, hi = dict(reserve=(-1, 3 * P if rng.random() < 0.7 else P * max_pages // 2), commit=(0, 3 * P), back=(-4 * P, 1),
                          drop=(DROP, DROP + 1))[what]
            rows = [(s, int(rng.integers(lo, hi))) for s in some[:1 + len(some) // 3 if what == "drop" else None]]
            call = "reserve" if what == "reserve" else "commit"
            getattr(c, call)(_i32([n for _, n in rows]), streams=_i32([s for s, _ in rows]))
            getattr(book, call)(rows)
        elif what == "fork":
            both = rng.permutation(n_streams)
            k = max(1, n_streams // 4)
            pairs = list(zip(rng.choice(both[k:], size=k).tolist(), both[:k].tolist()))
            c.fork(_i32([a for a, _ in pairs]), _i32([z for _, z in pairs]))
            book.fork(pairs)
        else:
            c.compact()
            book.compact()
        _same(c, book, content=step % 10 == 9)
        _whole(c)
