"""SamCache on the host: what it keeps and what it hands to the library, with stand-ins for the device."""
from __future__ import annotations

import pytest
import torch

import paper_2512_18337_b200 as S
from paper_2512_18337_b200 import binding


@pytest.fixture
def calls(monkeypatch):
    """Host tensors pass for device tensors; calls of the library are listed and not made."""
    made = []
    monkeypatch.setattr(binding, "_dev", lambda t: t if t is None or isinstance(t, int) else t.data_ptr())
    monkeypatch.setattr(binding.SamCache, "_rows", lambda self, t, heads: (t.data_ptr(), t.stride()[:3]))
    for name in ("sam_cache_init", "sam_cache_attend"):
        monkeypatch.setattr(binding, name, lambda *args, name=name: made.append((name, *args)))
    return made


def _cache(**kw):
    return S.SamCache(8, 16, 4, 4, 1, 2, 128, device="cpu", **kw)


@pytest.mark.parametrize("D", [64, 128])
def test_the_workspace_is_never_replaced(calls, D):
    """A recorded graph, or a call on another stream, may hold its address: a call with many query rows after one with a single
    row uses the same memory, and that memory is enough for every call."""
    c = S.SamCache(8, 16, 4, 4, 1, 2, D, device="cpu")
    used = set()
    for B, Q, H in ((1, 1, 2), (4, 64, 4), (2, 1, 8), (4, 3000, 2)):
        c.attend(0, torch.zeros(B, Q, H, D, dtype=torch.bfloat16))
        name, *_, workspace, size, _ = calls[-1]
        assert name == "sam_cache_attend" and size >= S.sam_cache_attend_workspace_bytes(c.handle, B, Q, H)
        used.add((workspace.data_ptr(), size))
    assert len(used) == 1
    assert not workspace.any()                             # zero-filled before the first call
    for B in (1, 300, 4096):
        for Q in (1, 2, 8, 9, 16, 17, 32, 33, 128, 129, 5000, 1 << 22):
            for H in (2, 8, 64):
                assert size >= S.sam_cache_attend_workspace_bytes(c.handle, B, Q, H)


def test_a_workspace_of_the_callers_is_used(calls):
    c = _cache()
    mine = torch.zeros(77, dtype=torch.int32)
    c.attend(0, torch.zeros(1, 1, 2, 128, dtype=torch.bfloat16), workspace=mine)
    assert calls[-1][-3] is mine and calls[-1][-2] == 308


def _books():
    return dict(page_table=torch.full((4, 4), -1, dtype=torch.int32), **{
        n: torch.zeros(size, dtype=torch.int32) for n, size in (("seq_len", 4), ("ref_count", 8), ("free_list", 8), ("meta", 4))})


@pytest.mark.parametrize("without", S.SamCache.BOOKS)
def test_books_given_in_part_are_refused(calls, without):
    """What is not given would be neither initialised nor in line with what is."""
    for names in ({without}, set(_books()) - {without}):
        with pytest.raises(ValueError, match="all together"):
            _cache(tensors={n: t for n, t in _books().items() if n in names})
    assert not calls


def test_unknown_tensors_are_refused(calls):
    with pytest.raises(ValueError, match="all together"):
        _cache(tensors=dict(_books(), pages_table=torch.zeros(4, 4, dtype=torch.int32)))
    with pytest.raises(ValueError, match="all together"):
        _cache(tensors=dict(seq_lens=torch.zeros(4, dtype=torch.int32)))


def test_books_given_are_kept_and_others_made(calls):
    given = _books()
    c = _cache(tensors=given)
    assert not calls and all(getattr(c, n) is t for n, t in given.items())
    pages = torch.zeros(8 * c.page_bytes, dtype=torch.uint8)
    for tensors in (None, {}, dict(pages=pages), dict(pages=pages, seq_len=None)):
        del calls[:]
        c = _cache(tensors=tensors)
        assert [x[0] for x in calls] == ["sam_cache_init"]
    assert c.pages is pages


def test_what_a_cache_allocates_belongs_to_its_stream(calls, monkeypatch):
    """The cache is emptied on the stream that it is made on: memory that another stream has just released, and may still be
    writing to, must not be under it."""
    made = []

    def empty(shape, dtype, device, stream, zero=False):
        made.append(stream)
        return torch.zeros(shape, dtype=dtype)
    monkeypatch.setattr(binding.SamCache, "_empty", staticmethod(empty))
    for name in ("empty", "zeros"):
        monkeypatch.setattr(torch, name, lambda *a, _make=getattr(torch, name), **kw: _make(*a, **kw) if "device" not in kw
                            else pytest.fail("allocated without the stream"))
    c = _cache(stream=1234)
    assert calls == [("sam_cache_init", c.handle, 1234)]
    assert made == [1234] * 8                              # pages, five books, scratch, workspace
