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
