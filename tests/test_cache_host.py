"""The 4-bit cache without a device: sizes, refusals, and the reference's own pins."""
from __future__ import annotations

import ctypes as C

import numpy as np
import pytest

from tests import cache_reference as R
import paper_2512_18337_b200 as S
from paper_2512_18337_b200.binding import _CacheStruct


def _struct(**over):
    f = dict(pages=128, page_table=4, seq_len=4, ref_count=4, free_list=4, meta=4, scratch=16, scratch_bytes=1 << 30, n_pages=8,
             page_tokens=16, n_streams=4, max_pages=4, n_layers=2, n_kv_heads=2, head_dim=128, k_exp=0, v_exp=0)
    f.update(over)
    return _CacheStruct(*(f[n] for n, _ in _CacheStruct._fields_))


def test_sizes():
    assert S.sam_cache_page_bytes(16, 1, 1, 128) == 2304
    assert S.sam_cache_page_bytes(64, 3, 8, 64) == 3 * 8 * 4 * 1152
    assert S.sam_cache_page_bytes(1024, 1000, 64, 128) == 1000 * 64 * 64 * 2304    # past 2^32
    for bad in ((8, 1, 1, 128), (24, 1, 1, 128), (2048, 1, 1, 128), (16, 0, 1, 128), (16, 1, 0, 128), (16, 1, 1, 96)):
        with pytest.raises(S.SamError) as e:
            S.sam_cache_page_bytes(*bad)
        assert e.value.status == -1
    assert S.sam_cache_scratch_bytes(4, 100) < S.sam_cache_scratch_bytes(4, 101)
    for bad in ((0, 1), (1, 0)):
        with pytest.raises(S.SamError):
            S.sam_cache_scratch_bytes(*bad)


BAD_CACHES = [dict(page_tokens=48), dict(head_dim=80), dict(n_pages=0), dict(n_streams=0), dict(max_pages=0),
              dict(max_pages=1 << 27), dict(max_pages=(1 << 26) + 1), dict(n_streams=1 << 20, max_pages=(1 << 10) + 1),
              dict(k_exp=25), dict(v_exp=-25), dict(page_table=0), dict(seq_len=0), dict(n_layers=0)]


@pytest.mark.parametrize("over", BAD_CACHES, ids=str)
def test_bad_caches_are_refused(over):
    lib = S.binding._load()
    c = C.addressof(s := _struct(**over))
    assert lib.sam_cache_init(c, None) == -1
    assert lib.sam_cache_reserve(c, 1, None, 16, None) == -1
    assert lib.sam_cache_commit(c, 1, None, 16, None) == -1
    assert lib.sam_cache_fork(c, 1, 16, 16, None) == -1
    assert lib.sam_cache_compact(c, None) == -1
    assert lib.sam_cache_copy_pages(c, c, 1, 16, 16, None) == -1
    assert lib.sam_cache_append(c, 0, 16, 16, 0, 0, 0, 0, 1, 1, None, None, None) == -1
    assert lib.sam_cache_read(c, 0, 1, 1, None, None, None, 16, 16, 0, None) == -1
    assert lib.sam_cache_attend_workspace_bytes(c, 1, 1, 2) == -1
    assert lib.sam_cache_attend(c, 0, 16, 0, 0, 0, 0, 1, 1, 2, None, None, 1.0, 0, 16, 0, 0, 0, None, 256, 1 << 30, None) == -1
    del s


def test_bad_arguments_are_refused():
    lib = S.binding._load()
    c = C.addressof(s := _struct())
    for name in ("sam_cache_init", "sam_cache_compact"):
        assert getattr(lib, name)(None, None) == -1
    # books and scratch
    for over, code in ((dict(ref_count=0), -1), (dict(meta=0), -1), (dict(free_list=0), -1), (dict(scratch=0), -1),
                       (dict(scratch=8), -1), (dict(scratch_bytes=64), -5)):
        d = C.addressof(t := _struct(**over))
        assert lib.sam_cache_commit(d, 1, None, 16, None) == code
        del t
    d = C.addressof(t := _struct(pages=64))
    assert lib.sam_cache_compact(d, None) == -1 and lib.sam_cache_append(d, 0, 16, 16, 0, 0, 0, 0, 1, 1, None, None, None) == -1
    # counts
    for call in (lambda B: lib.sam_cache_reserve(c, B, 16, 16, None), lambda B: lib.sam_cache_commit(c, B, 16, 16, None)):
        assert call(-1) == -1 and call(5) == -1 and call(5000) == -6 and call(0) == 0
    assert lib.sam_cache_reserve(c, 1, None, None, None) == -1 and lib.sam_cache_commit(c, 1, None, None, None) == -1
    assert lib.sam_cache_fork(c, 0, None, None, None) == 0 and lib.sam_cache_fork(c, 1, None, 16, None) == -1
    assert lib.sam_cache_fork(c, -1, 16, 16, None) == -1 and lib.sam_cache_fork(c, 5, 16, 16, None) == -1
    other = C.addressof(u := _struct(page_tokens=32))
    assert lib.sam_cache_copy_pages(c, other, 1, 16, 16, None) == -1 and lib.sam_cache_copy_pages(c, c, 1, None, 16, None) == -1
    assert lib.sam_cache_copy_pages(c, c, 0, None, None, None) == 0

    def append(layer=0, k=16, v=16, dtype=0, B=1, Q=1, streams=None):
        return lib.sam_cache_append(c, layer, k, v, dtype, 0, 0, 0, B, Q, streams, None, None)
    for over in (dict(layer=2), dict(layer=-1), dict(k=None), dict(v=None), dict(k=17), dict(dtype=2), dict(B=-1), dict(Q=-1), dict(B=5)):
        assert append(**over) == -1, over
    assert append(B=5000, streams=16) == -6 and append(B=0) == 0 and append(Q=0) == 0

    def read(layer=0, k=16, v=16, dtype=0, B=1, Q=1):
        return lib.sam_cache_read(c, layer, B, Q, None, None, None, k, v, dtype, None)
    for over in (dict(layer=2), dict(k=None), dict(v=8), dict(dtype=-1), dict(B=-1), dict(Q=-1), dict(B=5)):
        assert read(**over) == -1, over
    assert read(B=0) == 0

    need = lib.sam_cache_attend_workspace_bytes(c, 1, 1, 4)
    assert need > 0
    assert lib.sam_cache_attend_workspace_bytes(c, 1, 1, 3) == -1 and lib.sam_cache_attend_workspace_bytes(c, 5000, 1, 4) == -6

    def attend(layer=0, q=16, dtype=0, B=1, Q=1, H=4, window=0, out=16, lse=None, ws=256, ws_bytes=None):
        return lib.sam_cache_attend(c, layer, q, dtype, 0, 0, 0, B, Q, H, None, None, 1.0, window, out, 0, 0, 0, lse, ws,
                                    need if ws_bytes is None else ws_bytes, None)
    for over in (dict(layer=2), dict(q=None), dict(q=17), dict(dtype=5), dict(B=-1), dict(Q=-1), dict(H=3), dict(H=0), dict(window=-1),
                 dict(out=None), dict(lse=2), dict(ws=None), dict(ws=128), dict(B=5)):
        assert attend(**over) == -1, over
    assert attend(Q=1 << 30, ws_bytes=1 << 40) == -6
    one = C.addressof(w := _struct(n_kv_heads=1))
    assert lib.sam_cache_attend(one, 0, 16, 0, 0, 0, 0, 1, (1 << 30) + 1, 1, None, None, 1.0, 0, 16, 0, 0, 0, None, 256, 1 << 40, None) == -6
    assert attend(ws_bytes=need - 1) == -5 and attend(B=0) == 0 and attend(Q=0) == 0
    del s, u, w


def test_reference_rounds_to_the_nearest_value():
    """By brute force over all sixteen codes and all scales; ties go to the even code."""
    rng = np.random.default_rng(0)
    for exp in (0, -5, 3):
        x = rng.standard_normal((200, 16)) * 2.0 ** rng.integers(-8, 8, size=(200, 1))
        codes, scales = R.quantise(x, exp)
        s = R.E4M3[scales[:, 0]] * 2.0 ** exp
        want = np.abs(x).max(1) / 6
        assert (np.abs(s - want) <= np.abs(R.E4M3[:, None] * 2.0 ** exp - want).min(0) + 1e-18).all()
        got = R.values(codes, scales, exp)
        alt = np.concatenate([R.E2M1, -R.E2M1])[None, None] * s[:, None, None]
        assert (np.abs(got - x) <= np.abs(alt - x[..., None]).min(-1) + 1e-15).all()
    tie = np.array([[6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, 0]])
    codes, scales = R.quantise(tie, 0)
    assert R.values(codes, scales, 0)[0].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 0, -1, -1, -2, -2, -4, -4, 0]
    assert R.E4M3[-1] == 448 and R.E4M3[1] == 2.0 ** -9 and R.E4M3[8] == 2.0 ** -6


def test_reference_books_hold_together():
    """Whatever is done, counts equal the holders, and every page is held or on the free list once."""
    rng = np.random.default_rng(1)
    b = R.Books(60, 16, 6, 12)
    for _ in range(400):
        s = int(rng.integers(6))
        what = rng.integers(4)
        if what == 0:
            b.reserve([(s, int(rng.integers(1, 40)))])
        elif what == 1:
            b.commit([(s, int(rng.integers(-30, max(1, (b.table[s] >= 0).sum() * 16 - b.len[s] + 1))))])
        elif what == 2:
            b.fork([(s, int(rng.integers(6)))])
        else:
            b.compact()
        held = b.table[b.table >= 0]
        assert (np.bincount(held, minlength=60) == b.ref).all()
        assert sorted(b.free) == [p for p in range(60) if b.ref[p] == 0]
