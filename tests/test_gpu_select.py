"""Bounds of pages and the selection of blocks: equal, number by number, to the definition in whole numbers and fractions."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from tests import cache_reference as R
from tests.test_gpu_cache_attend import DEV, DT, _cache, _i32

pytestmark = pytest.mark.gpu


def _bounds(raw, D, k_exp):
    """codes [pages, layers, heads, 2, D], exps [pages, layers, heads] from the pages' bytes."""
    codes, scales = R.unpack_pages(raw, D)
    k = R.values(codes[0], scales[0], k_exp)                      # [pages, layers, heads, tokens, D]
    out = np.zeros((*k.shape[:3], 2, D), np.int8)
    exps = np.zeros(k.shape[:3], np.int8)
    for at in np.ndindex(*k.shape[:3]):
        x = k[at]
        if np.isnan(x).any():
            exps[at] = 127
            continue
        amax = np.abs(x).max()
        if amax == 0:
            continue
        e = -60
        while amax > 127 * 2.0 ** e:
            e += 1
        exps[at] = e
        out[at] = np.ceil(x.max(0) / 2.0 ** e), np.floor(x.min(0) / 2.0 ** e)
    return out, exps


@pytest.mark.parametrize("P,D,k_exp", [(16, 128, 0), (16, 64, -24), (32, 128, 24), (64, 64, 3), (1024, 128, -2)])
def test_rebuild(P, D, k_exp):
    rng = np.random.default_rng(P + D)
    c, raw, _ = _cache(rng, [3 * P, 1], [0, 0], P, 2, D, n_layers=3, k_exp=k_exp)
    raw[..., 16 * D:17 * D] = rng.integers(0, 0x7f, size=raw[..., 16 * D:17 * D].shape)   # every scale there is
    raw[0, 1, :, :, 16 * D:17 * D] = 0                                                     # a page of zeros
    raw[1, 0, 1, -1, 16 * D + 3] = 0xff                                                    # one of NaN
    c.pages.copy_(torch.from_numpy(raw))
    want, exps = _bounds(raw, D, k_exp)
    b = S.SamBounds(c)
    b.codes.fill_(55), b.exps.fill_(55)
    some = [2, -1, 0, 99, 0]
    b.rebuild(_i32(some))
    assert (b.codes[[0, 2]].cpu().numpy() == want[[0, 2]]).all() and (b.exps[[0, 2]].cpu().numpy() == exps[[0, 2]]).all()
    rest = [p for p in range(raw.shape[0]) if p not in (0, 2)]
    assert (b.codes[rest] == 55).all() and (b.exps[rest] == 55).all()
    b.rebuild()
    assert (b.codes.cpu().numpy() == want).all() and (b.exps.cpu().numpy() == exps).all()


@pytest.mark.parametrize("Q,P", [(1, 16), (17, 16), (100, 16), (40, 64), (3000, 16)])
def test_update(Q, P):
    """Exactly the pages that the new tokens fill up get bounds, in the one layer."""
    rng = np.random.default_rng(Q)
    lengths = [0, P - 1, P, 5 * P - 3, 7, 2 * P + 1]
    new = [Q, Q, Q, max(Q - 1, 0), -3, min(Q, 2)]
    c, raw, table = _cache(rng, lengths, [Q] * 6, P, 2, 128, garbage=False)
    table[2, 2:3] = -1
    c.page_table.copy_(torch.from_numpy(table))
    want, exps = _bounds(raw, 128, 0)
    b = S.SamBounds(c)
    b.codes.fill_(55), b.exps.fill_(55)
    streams = [3, 0, 5, 77, 1, 2, 4]
    b.update(1, Q, n_new=_i32([new[s] if s < 6 else Q for s in streams]), streams=_i32(streams))
    made = np.zeros(raw.shape[0], bool)
    for s in range(6):
        for i in range(lengths[s] // P, (lengths[s] + max(new[s], 0)) // P):
            if table[s, i] >= 0:
                made[table[s, i]] = True
    got, got_e = b.codes.cpu().numpy(), b.exps.cpu().numpy()
    assert (got[made, 1] == want[made, 1]).all() and (got_e[made, 1] == exps[made, 1]).all()
    assert (got[~made] == 55).all() and (got_e[~made] == 55).all() and (got[:, 0] == 55).all()


def _query_codes(q):
    """q [D] in 64 bits -> (whole numbers, power of two)."""
    q = np.where(np.isnan(q), 0, q)
    finite = np.abs(q[np.isfinite(q)])
    amax = finite.max() if finite.size else 0.0
    e = 0
    if amax >= 2.0 ** -126:
        e = -100
        while amax > 127 * 2.0 ** e:
            e += 1
    with np.errstate(over="ignore"):
        return np.clip(np.rint(q / 2.0 ** e), -127, 127).astype(int), e


def _select(q, n_new, lengths, table, codes, exps, g, P, share, n_sink, n_recent, n_blocks, layer):
    """q [B, Q, H, D] in 64 bits; rows without a stream have a length of None."""
    B, Q, H, D = q.shape
    Hkv = H // g
    out = -np.ones((B, -(-Q // share), Hkv, n_blocks), np.int32)
    for b in range(B):
        if lengths[b] is None:
            continue
        for l in range(out.shape[1]):
            rows = range(l * share, min((l + 1) * share, n_new[b], Q))
            if not rows:
                continue
            first, last = lengths[b] + rows[0], lengths[b] + rows[-1]
            for h in range(Hkv):
                x = [_query_codes(q[b, i, h * g + k]) for i in rows for k in range(g)]
                order = []
                for i in range(min(last // P + 1, len(table[b]))):
                    page = table[b][i]
                    if page < 0:
                        continue
                    if i < n_sink or i > first // P - n_recent:
                        rank = (0, 0.0)
                    elif exps[page, layer, h] == 127:
                        rank = (1, 0.0)
                    else:
                        hi, lo = codes[page, layer, h].astype(int)
                        with np.errstate(over="ignore"):
                            best = max(np.float32(np.maximum(w * hi, w * lo).sum()) * np.float32(2.0 ** e) for w, e in x)
                            rank = (2, -float(np.float32(best) * np.float32(2.0 ** float(exps[page, layer, h]))))
                    order.append((*rank, i))
                keep = sorted(i for *_, i in sorted(order)[:n_blocks])
                out[b, l, h, :len(keep)] = keep
    return out


def _run(rng, lengths, n_new, Q, H, Hkv, D, P, share, n_sink, n_recent, n_blocks, dtype="bf16", change=None, streams=None, holes=0.0, q=None):
    c, raw, table = _cache(rng, lengths, [Q] * len(lengths), P, Hkv, D, holes=holes, garbage=False)
    raw[..., 16 * D:17 * D] = rng.integers(0x28, 0x40, size=raw[..., 16 * D:17 * D].shape)
    if change:
        change(raw, table)
        c.pages.copy_(torch.from_numpy(raw))
        c.page_table.copy_(torch.from_numpy(table))
    else:
        c.pages.copy_(torch.from_numpy(raw))
    b = S.SamBounds(c)
    b.rebuild()
    rows = list(range(len(lengths))) if streams is None else streams
    if q is None:
        q = torch.from_numpy(rng.standard_normal((len(rows), Q, H, D)) * np.exp2(rng.integers(-3, 4, size=(len(rows), Q, H, 1))))
    q = q.to(DEV, DT[dtype])
    got = b.select(1, q, n_blocks, n_sink=n_sink, n_recent=n_recent, share=share, n_new=_i32(n_new), streams=None if streams is None else _i32(streams))
    codes, exps = _bounds(raw, D, 0)
    known = [0 <= s < len(lengths) for s in rows]
    want = _select(q.double().cpu().numpy(), n_new, [lengths[s] if ok else None for s, ok in zip(rows, known)],
                   [table[s] if ok else None for s, ok in zip(rows, known)], codes, exps, H // Hkv, P, share, n_sink, n_recent, n_blocks, 1)
    assert (got.cpu().numpy() == want).all()
    return c, b, q, got


CASES = [
    # lengths, n_new, Q, H, Hkv, D, P, share, n_sink, n_recent, n_blocks
    ([0], [1], 1, 1, 1, 64, 16, 1, 0, 1, 1),
    ([1000, 15, 16, 17, 300, 0], [1] * 6, 1, 8, 2, 128, 16, 1, 1, 2, 8),
    ([900, 33, 500], [5, 0, 3], 5, 7, 1, 128, 16, 1, 0, 1, 5),
    ([900, 33, 500], [17, 17, 4], 17, 8, 2, 64, 16, 17, 1, 2, 7),
    ([900, 5], [17, 9], 17, 12, 4, 128, 32, 5, 2, 3, 9),
    ([2100], [70], 70, 28, 4, 128, 16, 16, 1, 1, 12),
    ([640], [130], 130, 8, 1, 64, 16, 65, 0, 2, 20),           # 520 query rows a list
    ([5000, 4095, 4096], [2, 1, 2], 2, 16, 16, 64, 64, 2, 3, 4, 33),
    ([9000], [3], 3, 3, 1, 128, 1024, 3, 0, 1, 4),
    ([70000], [1], 1, 4, 1, 64, 16, 1, 1, 2, 64),              # more pages than fit shared memory
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_select(case, dtype):
    _run(np.random.default_rng(case), *CASES[case], dtype=dtype)


def test_equal_scores_go_to_the_lowest_block():
    """Pages with the same contents, a few distinct ones: whole classes tie."""
    def change(raw, table):
        for s in range(2):
            for i, p in enumerate(table[s][table[s] >= 0]):
                raw[p] = raw[table[s][i % 3]]
    for n_blocks in (3, 10, 25):
        _run(np.random.default_rng(1), [800, 799], [3, 3], 3, 8, 2, 128, 16, 3, 1, 1, n_blocks, change=change)


def test_queries_of_zero_list_the_first_blocks():
    q = torch.zeros(1, 1, 4, 128)
    q[..., ::2] = -0.0
    _, _, _, got = _run(np.random.default_rng(2), [500], [1], 1, 4, 1, 128, 16, 1, 1, 2, 6, q=q)
    assert got.flatten().tolist() == [0, 1, 2, 3, 30, 31]


def test_pages_with_nan_go_first_and_absent_ones_never():
    def change(raw, table):
        raw[table[0][20], 1, 0, 0, 16 * 128] = 0x7f
        raw[table[0][7], 1, 1, 0, 17 * 128 - 1] = 0xff
        table[0][[0, 5, 31, 33]] = -1
        table[1][:] = -1
    c, _, _, got = _run(np.random.default_rng(3), [540, 400], [2, 2], 2, 4, 2, 128, 16, 2, 1, 2, 6, change=change)
    got = got.cpu().numpy()
    assert 20 in got[0, 0, 0] and 7 in got[0, 0, 1] and (got[1] == -1).all()


@pytest.mark.parametrize("holes", [0.3, 0.9])
def test_holes_and_named_streams(holes):
    streams = [2, 99, 0, 1, -5]
    _run(np.random.default_rng(4), [700, 300, 1200], [9, 9, 4, 0, 9], 9, 6, 2, 128, 16, 4, 1, 2, 10, streams=streams, holes=holes)


def test_extreme_queries():
    """Sizes from the least to the largest, infinities and NaN among the channels."""
    rng = np.random.default_rng(5)
    q = rng.standard_normal((1, 8, 4, 128))
    for i, e in enumerate((100, 120, 126, -60, -99, -120, -133)):
        q[0, i] *= 2.0 ** e
    q[0, 7, :, 3], q[0, 7, :, 9], q[0, 7, 2, 50] = math.inf, math.nan, -math.inf
    _run(rng, [1000], [8], 8, 4, 2, 128, 16, 1, 0, 1, 9, q=torch.from_numpy(q))


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 3)])
def test_strided_queries(offset, pad):
    rng = np.random.default_rng(6)
    _, b, q, want = _run(rng, [400, 90], [5, 5], 5, 6, 2, 128, 16, 1, 1, 1, 6)
    flat = torch.zeros(offset + 2 * 6 * (5 * (128 + pad) + pad), dtype=q.dtype, device=DEV)
    qs = flat[offset:].as_strided(q.shape, (6 * (5 * (128 + pad) + pad), 128 + pad, 5 * (128 + pad) + pad, 1))
    qs.copy_(q)
    assert torch.equal(b.select(1, qs, 6, n_sink=1, n_recent=1), want)


def test_lists_beyond_one_launch():
    """More lists than the keys have room for at a time: the same lists."""
    rng = np.random.default_rng(8)
    c, b, q, want = _run(rng, [300, 250], [40, 33], 40, 2, 2, 64, 16, 1, 1, 1, 5)
    need = S.sam_cache_select_workspace_bytes(c.handle, 2, 40, 1)
    # a table of so many places that two lists fill the keys
    big = S.SamCache(c.pages.shape[0], 16, 2, 1 << 23, 2, 2, 64, 0, -3, device=DEV,
                     tensors=dict(pages=c.pages, **{n: getattr(c, n) for n in c.BOOKS if n != "page_table"},
                                  page_table=torch.full((2, 1 << 23), -1, dtype=torch.int32, device=DEV)))
    big.page_table[:, :c.page_table.shape[1]] = c.page_table
    assert need < S.sam_cache_select_workspace_bytes(big.handle, 2, 40, 1) == 1 << 27
    got = S.SamBounds(big, b.codes, b.exps).select(1, q, 5, n_sink=1, n_recent=1, n_new=_i32([40, 33]))
    assert torch.equal(got, want)
