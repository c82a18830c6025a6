"""Rotated appends, block selection, attention over blocks and shaped verification without a device: turns, sizes, refusals."""
from __future__ import annotations

import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from paper_2512_18337_b200 import binding
from paper_2512_18337_b200.binding import _RopeStruct, _ShapeStruct
from tests.test_cache_host import BAD_CACHES, _struct

# 2 pi to 60 digits
TWO_PI = Fraction(6283185307179586476925286766559005768394338798750211641949889, 10 ** 60)


@pytest.mark.parametrize("f", [1.0, 0.1, 1e-4 ** 0.7, 2.0 ** -40, 6.2, 100.25, -0.3, 0.0, 1e6])
def test_turns(f):
    """The fraction of a turn, off by 2^-64 of a unit or what a 64-bit mantissa of f / 2 pi leaves."""
    got = int(S.sam_rope_turns([f])[0])
    want = Fraction(f) / TWO_PI
    off = (Fraction(got, 1 << 64) - want) % 1
    off = min(off, 1 - off)
    assert off <= Fraction(3, 1 << 64) * max(1, math.ceil(abs(want)))


def test_turns_are_refused():
    lib = S.binding._load()
    f, t = (C.c_double * 65)(), (C.c_uint64 * 65)()
    assert lib.sam_rope_turns(f, 64, t) == 0
    for n in (0, -1, 65):
        assert lib.sam_rope_turns(f, n, t) == -1
    assert lib.sam_rope_turns(None, 1, t) == -1 and lib.sam_rope_turns(f, 1, None) == -1
    for bad in (math.nan, math.inf, -math.inf, 1.1e6):
        f[3] = bad
        assert lib.sam_rope_turns(f, 4, t) == -1 and lib.sam_rope_turns(f, 3, t) == 0


def _rope(**over):
    d = dict(turns=8, rotary_dim=128, interleaved=0, factor=1.0)
    d.update(over)
    return _RopeStruct(*(d[n] for n, _ in _RopeStruct._fields_))


@pytest.mark.parametrize("over", BAD_CACHES + [dict(pages=0), dict(pages=64)], ids=str)
def test_bad_caches_are_refused(over):
    lib, r = S.binding._load(), _rope()
    c = C.addressof(s := _struct(**over))
    assert lib.sam_cache_append_rotated(c, 0, 16, 0, 0, 0, 16, 16, 0, 0, 0, 16, 0, 0, 0, 0, C.addressof(r), 1, 1, 2, None, None, None, None) == -1
    assert lib.sam_cache_bounds_update(c, 0, 16, 16, 1, 1, None, None, None) == -1
    assert lib.sam_cache_bounds_rebuild(c, 16, 16, 1, None, None) == -1
    assert lib.sam_cache_select(c, 0, 16, 16, 16, 0, 0, 0, 0, 1, 1, 2, None, None, 1, 0, 1, 16, 4, 256, 1 << 30, None) == -1
    assert lib.sam_cache_attend_blocks(c, 0, 16, 0, 0, 0, 0, 1, 1, 2, None, None, 16, 4, 1, 1.0, 16, 0, 0, 0, None, 256, 1 << 30, None) == -1
    if "pages" not in over:
        assert lib.sam_cache_select_workspace_bytes(c, 1, 1, 1) == -1
        assert lib.sam_cache_attend_blocks_workspace_bytes(c, 1, 1, 2, 1) == -1
    del s


def test_append_rotated_refuses():
    lib = S.binding._load()
    c = C.addressof(s := _struct())

    def call(layer=0, q=16, k=16, v=16, out=16, dtype=0, rope=None, B=1, Q=1, H=2, streams=None, positions=None, **turn):
        r = _rope(**turn)
        return lib.sam_cache_append_rotated(c, layer, q, 0, 0, 0, k, v, 0, 0, 0, out, 0, 0, 0, dtype, rope or C.addressof(r), B, Q, H, streams, None,
                                            positions, None)
    for over in (dict(layer=2), dict(layer=-1), dict(q=None), dict(q=17), dict(k=None), dict(v=None), dict(v=1), dict(out=None), dict(out=3), dict(dtype=2),
                 dict(B=-1), dict(Q=-1), dict(H=-1), dict(B=5), dict(positions=2), dict(turns=None), dict(turns=12), dict(rotary_dim=0),
                 dict(rotary_dim=16), dict(rotary_dim=48), dict(rotary_dim=160), dict(factor=math.nan), dict(factor=math.inf)):
        assert call(**over) == -1, over
    assert lib.sam_cache_append_rotated(c, 0, 16, 0, 0, 0, 16, 16, 0, 0, 0, 16, 0, 0, 0, 0, None, 1, 1, 2, None, None, None, None) == -1
    assert call(B=5000, streams=16) == -6 and call(H=16385) == -6 and call(Q=(1 << 30) + 1) == -6 and call(B=3, Q=1 << 30) == -6
    assert call(B=0) == 0 and call(Q=0) == 0
    small = C.addressof(t := _struct(head_dim=64))
    r = _rope()
    assert lib.sam_cache_append_rotated(small, 0, 16, 0, 0, 0, 16, 16, 0, 0, 0, 16, 0, 0, 0, 0, C.addressof(r), 1, 1, 2, None, None, None, None) == -1
    del s, t


def test_bounds_and_select_refuse():
    lib = S.binding._load()
    c = C.addressof(s := _struct())
    for over in (dict(layer=2), dict(codes=None), dict(codes=8), dict(exps=None), dict(B=-1), dict(Q=-1), dict(B=5)):
        d = dict(layer=0, codes=16, exps=1, B=1, Q=1)
        d.update(over)
        assert lib.sam_cache_bounds_update(c, d["layer"], d["codes"], d["exps"], d["B"], d["Q"], None, None, None) == -1, over
    assert lib.sam_cache_bounds_update(c, 0, 16, 1, 0, 1, None, None, None) == 0
    assert lib.sam_cache_bounds_rebuild(c, 16, 1, -1, None, None) == -1 and lib.sam_cache_bounds_rebuild(c, 16, 1, 9, None, None) == -1
    assert lib.sam_cache_bounds_rebuild(c, None, 1, 1, None, None) == -1 and lib.sam_cache_bounds_rebuild(c, 16, 1, 0, None, None) == 0
    need = lib.sam_cache_select_workspace_bytes(c, 2, 5, 2)
    assert need == 2 * (3 + 2) * 2 * 4 * 4                                         # lists of two rows, some to spare, heads, pages
    wide = C.addressof(w := _struct(max_pages=1 << 16, n_kv_heads=8))
    assert lib.sam_cache_select_workspace_bytes(wide, 64, 2048, 1) == 1 << 27      # as much as is in flight at a time
    huge = C.addressof(h := _struct(max_pages=1 << 26, n_streams=1, n_kv_heads=8))
    assert lib.sam_cache_select_workspace_bytes(huge, 1, 1, 1) == 1 << 31          # one list at least
    assert lib.sam_cache_select_workspace_bytes(c, 1, 1, 0) == -1 and lib.sam_cache_select_workspace_bytes(c, 5000, 1, 1) == -6

    def select(layer=0, codes=16, exps=1, q=16, dtype=0, B=1, Q=5, H=4, share=2, n_sink=0, n_recent=1, blocks=16, n_blocks=4, ws=256, ws_bytes=need):
        return lib.sam_cache_select(c, layer, codes, exps, q, dtype, 0, 0, 0, B, Q, H, None, None, share, n_sink, n_recent, blocks, n_blocks, ws,
                                    ws_bytes, None)
    for over in (dict(layer=-1), dict(codes=None), dict(codes=4), dict(exps=None), dict(q=None), dict(q=1), dict(dtype=7), dict(B=-1), dict(Q=-1), dict(H=3),
                 dict(H=0), dict(share=0), dict(n_sink=-1), dict(n_recent=0), dict(blocks=None), dict(blocks=2), dict(n_blocks=0), dict(ws=None), dict(ws=128),
                 dict(n_sink=3), dict(n_recent=4), dict(n_blocks=1), dict(B=5)):
        assert select(**over) == -1, over
    # a run of 5 tokens of pages of 16 lies in up to two blocks, one of 19 in up to three
    assert select(share=5, n_sink=1, n_recent=2, n_blocks=3) == -1
    assert select(share=19, Q=19, n_sink=0, n_recent=1, n_blocks=2, ws_bytes=0) == -1
    assert select(share=19, Q=19, n_sink=0, n_recent=1, n_blocks=3, ws_bytes=0) == -5
    assert select(ws_bytes=16) == -5 and select(B=0) == 0 and select(Q=0) == 0
    del s, w, h


def test_attend_blocks_refuses():
    lib = S.binding._load()
    c = C.addressof(s := _struct())
    need = lib.sam_cache_attend_blocks_workspace_bytes(c, 1, 5, 4, 2)
    assert need == lib.sam_cache_attend_workspace_bytes(c, 1, 2, 4)
    assert lib.sam_cache_attend_blocks_workspace_bytes(c, 1, 5, 4, 0) == -1 and lib.sam_cache_attend_blocks_workspace_bytes(c, 1, 5, 3, 1) == -1

    def call(layer=0, q=16, dtype=0, B=1, Q=5, H=4, blocks=16, n_blocks=4, share=2, scale=1.0, out=16, lse=None, ws=256, ws_bytes=need):
        return lib.sam_cache_attend_blocks(c, layer, q, dtype, 0, 0, 0, B, Q, H, None, None, blocks, n_blocks, share, scale, out, 0, 0, 0, lse, ws, ws_bytes, None)
    for over in (dict(layer=2), dict(q=None), dict(q=17), dict(dtype=5), dict(B=-1), dict(Q=-1), dict(H=3), dict(H=0), dict(blocks=None), dict(blocks=2),
                 dict(n_blocks=0), dict(share=0), dict(scale=math.nan), dict(scale=math.inf), dict(out=None), dict(out=1), dict(lse=2), dict(ws=None),
                 dict(ws=128), dict(B=5)):
        assert call(**over) == -1, over
    assert call(Q=1 << 30, ws_bytes=1 << 40) == -6 and call(ws_bytes=need - 1) == -5 and call(B=0) == 0 and call(Q=0) == 0
    del s


def _shape(**over):
    d = dict.fromkeys((n for n, _ in _ShapeStruct._fields_), None)
    d.update(counts=4, seen=4, n_streams=4, max_bias=0, n_masks=0)
    d.update(over)
    return _ShapeStruct(*(d[n] for n, _ in _ShapeStruct._fields_))


def test_shaped_verification_refuses():
    lib = S.binding._load()

    def call(logits=16, stride=100, B=2, K=3, V=100, drafts=16, streams=None, keys=8, shape=None, **over):
        s = _shape(**over)
        return lib.sam_argmax_shaped(logits, stride, B, K, V, drafts, streams, C.addressof(s), keys, None)
    for over in (dict(logits=None), dict(logits=1), dict(stride=99), dict(B=-1), dict(K=0), dict(K=33), dict(V=0), dict(V=(1 << 30) + 1, stride=1 << 40), dict(drafts=None),
                 dict(keys=None), dict(keys=4), dict(counts=None), dict(seen=None), dict(counts=2), dict(n_streams=0), dict(n_streams=-1),
                 dict(B=5), dict(max_bias=-1), dict(max_bias=1), dict(max_bias=1, bias_tokens=4), dict(n_masks=-1),
                 dict(masks=4), dict(mask_of=4), dict(masks=4, mask_of=4), dict(masks=2, mask_of=4, n_masks=1)):
        assert call(**over) == -1, over
    assert lib.sam_argmax_shaped(16, 100, 2, 3, 100, 16, None, None, 8, None) == -1
    assert call(B=0) == 0 and call(max_bias=513, bias_tokens=4, bias_values=4) == -6

    def verify(keys=8, B=1, K=3, drafts=4, n_draft=4, argmax=4, accepted=4, n_accepted=4, values=None):
        return lib.sam_verify_from_keys(keys, B, K, drafts, n_draft, argmax, accepted, n_accepted, values, None)
    for over in (dict(keys=None), dict(keys=4), dict(B=-1), dict(K=0), dict(K=33), dict(drafts=None), dict(n_draft=None), dict(argmax=None),
                 dict(accepted=None), dict(n_accepted=None), dict(values=2)):
        assert verify(**over) == -1, over
    assert verify(B=0) == 0


def test_history_refuses():
    lib = S.binding._load()

    def add(counts=4, seen=4, n_streams=4, V=100, B=1, streams=None, tokens=4, ld=5):
        return lib.sam_history_add(counts, seen, n_streams, V, B, streams, tokens, ld, None, 0, None)
    for over in (dict(counts=None), dict(seen=None), dict(counts=2), dict(seen=1), dict(n_streams=0), dict(V=0), dict(V=(1 << 30) + 1), dict(B=-1), dict(B=5), dict(tokens=None),
                 dict(ld=-1)):
        assert add(**over) == -1, over
    assert add(B=65536, streams=4) == -6 and add(B=0) == 0 and add(ld=0) == 0

    def copy(counts=4, seen=4, n_streams=4, V=100, n=1, src=4, dst=4):
        return lib.sam_history_copy(counts, seen, n_streams, V, n, src, dst, None)
    for over in (dict(counts=None), dict(seen=None), dict(n_streams=0), dict(V=0), dict(n=-1), dict(n=5), dict(dst=None)):
        assert copy(**over) == -1, over
    assert copy(n=65536, n_streams=1 << 20) == -6 and copy(n=0) == 0


# ------------------------------------------------------------------ the Python objects, with stand-ins for the device
@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(binding, "_dev", lambda t: t if t is None or isinstance(t, int) else t.data_ptr())
    monkeypatch.setattr(binding.SamCache, "_rows", lambda self, t, heads: (t.data_ptr(), t.stride()[:3]))
    for name in ("sam_cache_init", "sam_cache_append_rotated", "sam_cache_attend_blocks", "sam_cache_select", "sam_cache_bounds_update",
                 "sam_cache_bounds_rebuild"):
        monkeypatch.setattr(binding, name, lambda *args, name=name: made.append((name, *args)))
    return made


def test_objects_check_what_they_are_given(calls):
    c = S.SamCache(8, 16, 4, 4, 1, 2, 128, device="cpu")
    rope = S.SamRope(np.ones(64), device="cpu")
    q, k = torch.zeros(2, 3, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 3, 2, 128, dtype=torch.bfloat16)
    assert c.append_rotated(0, q, k, k.clone(), rope, out=q) is q and calls[-1][0] == "sam_cache_append_rotated"
    assert c.append_rotated(0, q, k, k.clone(), rope).shape == q.shape
    for bad in (dict(q=q.half()), dict(q=q[:, :2]), dict(v=k[:1]), dict(v=k.half()), dict(out=q[:1]), dict(positions=torch.zeros(2, 3)),
                dict(positions=torch.zeros(2, 2, dtype=torch.int32)), dict(n_new=torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            c.append_rotated(0, bad.pop("q", q), k, bad.pop("v", k), rope, **bad)
    bounds = S.SamBounds(c)
    assert bounds.codes.shape == (8, 1, 2, 2, 128) and bounds.exps.shape == (8, 1, 2)
    for bad in (dict(codes=bounds.codes[:4]), dict(exps=bounds.exps.short())):
        with pytest.raises(ValueError):
            S.SamBounds(c, **bad)
    blocks = bounds.select(0, q, 4, share=2)
    assert blocks.shape == (2, 2, 2, 4) and blocks.dtype == torch.int32 and calls[-1][0] == "sam_cache_select"
    with pytest.raises(ValueError):
        bounds.select(0, q, 4, share=2, out=blocks[:, :1])
    out, lse = c.attend_blocks(0, q, blocks, share=2)
    assert out.shape == q.shape and lse.shape == (2, 3, 4) and calls[-1][0] == "sam_cache_attend_blocks"
    for bad in (dict(share=1), dict(share=0), dict(blocks=blocks.long()), dict(blocks=blocks[..., 0]), dict(out=q[:1]), dict(lse=lse.double())):
        with pytest.raises(ValueError):
            c.attend_blocks(0, q, bad.pop("blocks", blocks), share=bad.pop("share", 2), **bad)
    bounds.rebuild()
    assert calls[-1][0] == "sam_cache_bounds_rebuild" and calls[-1][4] == 8
    bounds.update(0, 3, n_new=torch.zeros(2, dtype=torch.int32))
    assert calls[-1][0] == "sam_cache_bounds_update" and calls[-1][5:7] == (2, 3)


def test_shapes_check_what_they_are_given(calls):
    i32 = dict(dtype=torch.int32)
    counts, seen = torch.zeros(2, 70, **i32), torch.zeros(2, 3, **i32)
    ok = dict(counts=counts, seen=seen, repetition=torch.ones(2), bias_tokens=torch.zeros(2, 4, **i32), bias_values=torch.zeros(2, 4),
              n_bias=torch.zeros(2, **i32), masks=torch.zeros(5, 3, **i32), mask_of=torch.zeros(2, 4, **i32))
    s = S.SamShape(70, **ok)
    assert (s._struct.n_streams, s._struct.max_bias, s._struct.n_masks) == (2, 4, 5) and s.check(2, 3, 70) == s.handle
    for bad in (dict(counts=None), dict(seen=seen[:, :2]), dict(counts=counts.long()), dict(seen=seen[:1]), dict(repetition=torch.ones(2, 1)),
                dict(repetition=torch.ones(2).double()), dict(bias_values=None), dict(bias_values=torch.zeros(2, 3)), dict(masks=torch.zeros(5, 2, **i32)),
                dict(mask_of=None), dict(n_bias=torch.zeros(2))):
        with pytest.raises(ValueError):
            S.SamShape(70, **{**ok, **bad})
    for B, K, V in ((3, 3, 70), (2, 4, 70), (2, 3, 71)):
        with pytest.raises(ValueError):
            s.check(B, K, V)
    h = S.SamHistory(3, 70, device="cpu")
    assert h.counts.shape == (3, 70) and h.seen.shape == (3, 3) and not h.counts.any()
    for bad in (torch.zeros(3, **i32), torch.zeros(3, 2)):
        with pytest.raises(ValueError):
            h.add(bad)
    with pytest.raises(ValueError):
        h.add(torch.zeros(2, 2, **i32), n=torch.zeros(3, **i32))
