"""Reserving, committing, forking, compacting and copying pages, against lists that one row after the other changes."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from tests import cache_reference as R
import paper_2512_18337_b200 as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _pair(n_pages, P, n_streams, max_pages, seed=0, layers=2, Hkv=1, D=64):
    rng = np.random.default_rng(seed)
    c = S.SamCache(n_pages, P, n_streams, max_pages, layers, Hkv, D, device=DEV)
    raw = rng.integers(0, 256, size=tuple(c.pages.shape), dtype=np.uint8)
    c.pages.copy_(torch.from_numpy(raw))
    return c, R.Books(n_pages, P, n_streams, max_pages, raw.reshape(n_pages, -1).copy()), rng


def _same(c, book, content=True):
    n_free, status = c.status()
    assert status == book.status
    assert n_free == len(book.free)
    assert c.free_list[:n_free].tolist() == book.free
    assert (c.page_table.cpu().numpy() == book.table).all()
    assert (c.ref_count.cpu().numpy() == book.ref).all()
    assert (c.seq_len.cpu().numpy() == book.len).all()
    if content:
        assert (c.pages.view(len(book.ref), -1).cpu().numpy() == book.pages).all()


@pytest.mark.parametrize("P,n_streams,max_pages,n_pages", [(16, 1, 3, 4), (16, 7, 9, 64), (32, 40, 6, 200), (64, 300, 5, 1300),
                                                           (16, 1500, 4, 5000), (16, 33, 90, 2500)])
def test_random_walk(P, n_streams, max_pages, n_pages):
    """Long mixed sequences of all calls, full pools and full tables among them."""
    c, book, rng = _pair(n_pages, P, n_streams, max_pages, seed=P + n_streams)
    _same(c, book)
    for step in range(40):
        what = rng.choice(["reserve", "reserve", "reserve", "commit", "commit", "fork", "back", "drop", "compact"])
        some = rng.permutation(n_streams)[:rng.integers(1, n_streams + 1)]
        named = rng.random() < 0.5
        if not named:
            some = np.arange(len(some))
        streams = _i32(some) if named else None
        if what == "reserve":
            n = rng.integers(-1, 2 * P, size=len(some))
            if rng.random() < 0.3:      # write at once: the lengths move on with it
                n = np.minimum(n, P)
            c.reserve(_i32(n), streams=streams)
            book.reserve(list(zip(some.tolist(), n.tolist())))
        elif what in ("commit", "back", "drop"):
            lo, hi = {"commit": (0, P), "back": (-3 * P, 1), "drop": (-(1 << 31), -(1 << 31) + 1)}[what]
            n = rng.integers(lo, hi, size=len(some))
            # no further than the pages that are there
            room = np.array([(book.table[s] >= 0).sum() * P - book.len[s] for s in some])
            n = np.minimum(n, room)
            c.commit(_i32(n), streams=streams)
            book.commit(list(zip(some.tolist(), n.tolist())))
        elif what == "fork" and n_streams > 1:
            both = rng.permutation(n_streams)
            k = max(1, n_streams // 3)
            src = rng.choice(both[k:], size=k) if rng.random() < 0.5 else np.repeat(both[k], k)
            c.fork(_i32(src), _i32(both[:k]))
            book.fork(list(zip(src.tolist(), both[:k].tolist())))
        elif what == "compact":
            c.compact()
            book.compact()
        _same(c, book, content=step % 8 == 7 or n_pages < 100)
    _same(c, book)


@pytest.mark.parametrize("P", [16, 64])
def test_reserving_for_prompts(P):
    """Rows that need hundreds of pages beside rows that need none or one; holes in a table are filled; shared ends are copied."""
    c, book, rng = _pair(7000 if P == 16 else 2000, P, 9, 3000, seed=P, layers=1)
    for step, n in enumerate(([0, 20000, 3, 150, 17 * P, 0, 1, 30001, 8 * P], [40, 5, 0, 2500, 9 * P, 100, 0, 77, 12 * P])):
        c.reserve(_i32(n))
        book.reserve(list(enumerate(n)))
        _same(c, book, content=False)
        keep = [x if i != 3 else x // 2 for i, x in enumerate(n)]
        c.commit(_i32(keep))
        book.commit(list(enumerate(keep)))
        _same(c, book, content=False)
        if step == 0:
            c.fork(_i32([1, 3]), _i32([0, 5]))
            book.fork([(1, 0), (3, 5)])
    c.reserve(_i32([20 * P, 20 * P]), streams=_i32([1, 3]))
    book.reserve([(1, 20 * P), (3, 20 * P)])
    _same(c, book)
    # absent pages in the middle of what is reserved
    c.page_table[1, 1 + int(book.len[1]) // P + 4] = -1
    book.table[1, 1 + int(book.len[1]) // P + 4] = -1
    c.reserve(_i32([30 * P, 1]), streams=_i32([1, 8]))
    book.reserve([(1, 30 * P), (8, 1)])
    assert (c.page_table.cpu().numpy() == book.table).all()


def test_copy_on_write_and_the_last_holder():
    """Three holders of a half-filled page: writers get copies, unless all write: then the last keeps it."""
    c, book, _ = _pair(20, 16, 4, 3)
    for b in (c, book):
        args = (lambda r: r) if b is book else (lambda r: _i32([n for _, n in r]))
        rows = [(0, 24), (1, 0), (2, 0), (3, 0)]
        b.reserve(args(rows))
        b.commit(args(rows))
    c.fork(_i32([0, 0]), _i32([1, 2]))
    book.fork([(0, 1), (0, 2)])
    _same(c, book)
    assert c.ref_count.max() == 3
    c.reserve(_i32([1, 1, 0, 0]))
    book.reserve([(0, 1), (1, 1)])
    _same(c, book)
    c.reserve(_i32([2, 0]), streams=_i32([2, 3]))
    book.reserve([(2, 2)])
    _same(c, book)
    assert (c.ref_count.cpu().numpy() <= 3).all()


def test_all_holders_write():
    c, book, _ = _pair(20, 16, 4, 3, seed=2)
    c.reserve(_i32([0, 0, 5, 0]))
    book.reserve([(2, 5)])
    c.commit(_i32([0, 0, 5, 0]))
    book.commit([(2, 5)])
    c.fork(_i32([2, 2, 2]), _i32([3, 0, 1]))
    book.fork([(2, 3), (2, 0), (2, 1)])
    c.reserve(_i32([1, 1, 1, 1]), streams=_i32([3, 0, 2, 1]))
    book.reserve([(3, 1), (0, 1), (2, 1), (1, 1)])
    _same(c, book)


def test_too_few_pages_changes_nothing_but_the_status():
    c, book, _ = _pair(5, 16, 3, 8, seed=3)
    for rows in ([40, 8, 0], [0, 0, 33], [16 * 9, 0, 0]):
        c.reserve(_i32(rows))
        book.reserve(list(enumerate(rows)))
        _same(c, book)
    assert c.status()[1] == S.SAM_CACHE_OUT_OF_PAGES | S.SAM_CACHE_TABLE_FULL
    # also with shared pages that would have been copied
    c.commit(_i32([40, 8, 0]))
    book.commit([(0, 40), (1, 8)])
    c.fork(_i32([1]), _i32([2]))
    book.fork([(1, 2)])
    for rows in ([0, 1, 17], [0, 25, 25]):
        c.reserve(_i32(rows))
        book.reserve(list(enumerate(rows)))
        _same(c, book)


def test_fork_refusals():
    c, book, _ = _pair(8, 16, 3, 4, seed=4)
    c.reserve(_i32([20, 1, 0]))
    book.reserve([(0, 20), (1, 1)])
    c.commit(_i32([20, 0, 0]))
    book.commit([(0, 20), (1, 0)])
    c.fork(_i32([0, 0, 0, -1])[:3], _i32([1, 0, 7]))
    book.fork([(0, 1), (0, 0), (0, 7)])
    # stream 1 holds a page without tokens no more: the commit gave it back
    _same(c, book)
    assert c.status()[1] == S.SAM_CACHE_BAD_FORK


def test_copy_pages_between_pools():
    a, _, rng = _pair(9, 32, 2, 4, seed=5, layers=3, Hkv=2, D=128)
    b, _, _ = _pair(6, 32, 2, 4, seed=6, layers=3, Hkv=2, D=128)
    before = b.pages.clone()
    a.copy_pages(b, _i32([8, 0, 4, -1, 9, 2]), _i32([1, 5, 0, 2, 3, 6]))
    want = before
    for f, t in ((8, 1), (0, 5), (4, 0)):
        want[t] = a.pages[f]
    assert torch.equal(b.pages, want)
    mine = a.pages.clone()
    a.copy_pages(a, _i32([3]), _i32([7]))
    mine[7] = mine[3]
    assert torch.equal(a.pages, mine)


def test_bad_ids_in_the_table_are_no_pages():
    """Entries out of range (a table that the caller filled) are read as absent, not followed."""
    c = S.SamCache(4, 16, 2, 2, 1, 1, 64, device=DEV)
    c.page_table.copy_(_i32([[77, -5], [1, 1 << 30]]))
    c.seq_len.copy_(_i32([30, 20]))
    kv = torch.ones(2, 4, 1, 64, dtype=torch.bfloat16, device=DEV)
    c.append(0, kv, kv)
    k, _ = c.read(0, max_n=32)
    assert (k[0] == 0).all() and (k[1, 16:] == 0).all()
    out, lse = c.attend(0, kv)
    assert (out[0] == 0).all() and torch.isneginf(lse[0]).all() and torch.isfinite(lse[1]).all()


def test_pages_in_a_graph():
    c, book, _ = _pair(64, 16, 4, 12, seed=8)
    n, keep = _i32([9, 0, 3, 16]), _i32([5, 0, 3, 2])
    c.reserve(n)
    c.commit(keep)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.reserve(n)
        c.commit(keep)
    for _ in range(4):
        g.replay()
    torch.cuda.synchronize()
    for _ in range(5):
        book.reserve(list(enumerate([9, 0, 3, 16])))
        book.commit(list(enumerate([5, 0, 3, 2])))
    _same(c, book)
