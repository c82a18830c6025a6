"""Attention over the 4-bit cache, and keys and values into and out of it, against 64-bit numpy."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from tests import cache_reference as R
import paper_2512_18337_b200 as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
BITS = {"bf16": 8, "fp16": 11}


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _cache(rng, lengths, extra, P, Hkv, D, n_layers=2, k_exp=0, v_exp=-3, max_pages=None, holes=0.0, garbage=True):
    """A cache of random codes over shuffled pages; what lies behind the last token is 0xFF (a NaN scale)."""
    held = [-(-(l + e) // P) for l, e in zip(lengths, extra)]
    max_pages = max_pages or max(max(held), 1)
    n_pages = sum(held) + 2
    raw = rng.integers(0, 256, size=(n_pages, n_layers, Hkv, P // 16, 18 * D), dtype=np.uint8)
    raw[..., 16 * D:] = rng.integers(0x20, 0x38, size=raw[..., 16 * D:].shape)
    order = rng.permutation(n_pages)
    table = -np.ones((len(lengths), max_pages), np.int32)
    at = 0
    for s, n in enumerate(held):
        table[s, :n] = order[at:at + n]
        at += n
        end = lengths[s] + extra[s]
        if garbage and n and end % P:
            page = raw[order[at - 1]].reshape(n_layers, Hkv, P // 16, 18 * D)
            for t in range(end % P, P):
                for part, width in ((0, D // 2), (8 * D, D // 2), (16 * D, D // 16), (17 * D, D // 16)):
                    o = part + (t % 16) * width
                    page[:, :, t // 16, o:o + width] = 0xFF
    if holes:
        table[rng.random(table.shape) < holes] = -1
    c = S.SamCache(n_pages, P, len(lengths), max_pages, n_layers, Hkv, D, k_exp, v_exp, device=DEV)
    c.pages.copy_(torch.from_numpy(raw))
    c.page_table.copy_(torch.from_numpy(table))
    c.seq_len.copy_(_i32(lengths))
    return c, raw, table


def _tokens(raw, table, row, layer, P, D, exps):
    """Keys and values [T, Hkv, D] of a stream, and which positions have a page."""
    codes, scales = R.unpack_pages(raw, D)
    pages = table[row]
    out = [R.values(codes[w][np.maximum(pages, 0), layer].transpose(0, 2, 1, 3).reshape(-1, raw.shape[2], D),
                    scales[w][np.maximum(pages, 0), layer].transpose(0, 2, 1, 3).reshape(-1, raw.shape[2], D // 16), exps[w])
           for w in range(2)]
    return (*out, np.repeat(pages >= 0, P))


def _check(out, lse, ref, dtype, D):
    """Per element: weights rounded to 11 bits (2^-11 of the mean of |v|; their sum is not rounded); products of 32-bit
    sums, which shift an exponent by at most (D + 8) 2^-24 of the terms' size, in numerator and denominator; a few operations
    more; and half the spacing of the result's type (of fp16's subnormals at least) where that leaves it."""
    o, l, mean_abs, size = ref
    shift = (D + 8) * 2.0 ** -24 * size + 2.0 ** -20
    before = (2.0 ** -11 + 2 * shift)[..., None] * mean_abs + 2.0 ** -30
    e = np.floor(np.log2(np.abs(o) + before))
    bound = before + np.maximum(2.0 ** (e - BITS[dtype]), 2.0 ** -25)
    out = out.double().cpu().numpy()
    bad = np.abs(out - o) > bound
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(out - o).max(), bound[bad][:4])
    lse = lse.double().cpu().numpy()
    dead = np.isinf(l)
    assert (np.isneginf(lse) == dead).all()
    assert (out[dead] == 0).all()
    assert (np.abs(lse[~dead] - l[~dead]) <= shift[~dead] + 2.0 ** -21 * (1 + np.abs(l[~dead]))).all()


CASES = [
    # lengths, n_new, Q, H, Hkv, D, P, window
    ([0], [1], 1, 1, 1, 64, 16, 0),
    ([0, 1, 15, 16, 17], [1, 1, 1, 1, 1], 1, 8, 2, 128, 16, 0),
    ([5, 0, 100, 33], [0, 3, 5, -2], 5, 6, 2, 128, 16, 0),
    ([63, 64, 65, 127, 128, 129], [2, 1, 2, 1, 2, 1], 2, 7, 1, 64, 64, 0),
    ([300, 31], [17, 17], 17, 8, 2, 128, 32, 0),
    ([300, 31], [17, 4], 17, 8, 1, 128, 16, 0),
    ([700], [33], 33, 10, 2, 128, 16, 0),
    ([257, 5], [9, 9], 9, 28, 4, 64, 128, 0),
    ([700, 40], [1, 1], 1, 16, 16, 64, 16, 100),
    ([700, 40, 3], [17, 9, 1], 17, 5, 1, 128, 16, 37),
    ([500], [17], 17, 4, 4, 128, 256, 1),
    ([40], [150], 150, 4, 2, 128, 16, 0),
    ([0], [129], 129, 9, 3, 64, 16, 0),
    ([1000], [1], 1, 64, 1, 128, 16, 0),
    ([4000], [1], 1, 3, 1, 64, 1024, 0),
    ([211], [300], 300, 2, 1, 128, 32, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attend(case, dtype):
    lengths, n_new, Q, H, Hkv, D, P, window = CASES[case]
    rng = np.random.default_rng(100 + case)
    c, raw, table = _cache(rng, lengths, [max(n, 0) for n in n_new], P, Hkv, D)
    q = torch.from_numpy(rng.standard_normal((len(lengths), Q, H, D))).to(DEV, DT[dtype])
    for layer, scale in ((0, None), (1, 0.31)):
        out, lse = c.attend(layer, q, n_new=_i32(n_new), scale=scale, window=window)
        for b in range(len(lengths)):
            k, v, there = _tokens(raw, table, b, layer, P, D, (0, -3))
            ref = R.attend(q[b].double().cpu().numpy(), k, v, there, lengths[b], n_new[b], H // Hkv,
                           D ** -0.5 if scale is None else scale, window)
            _check(out[b], lse[b], ref, dtype, D)


@pytest.mark.parametrize("Q,H,Hkv,D", [(1, 8, 2, 128), (17, 8, 1, 128), (40, 8, 2, 64)])
def test_attend_absent_pages_and_named_streams(Q, H, Hkv, D):
    """Pages that are not there are not seen; whole rows can lose everything; rows name their streams in any order, and an
    unknown stream reads as nothing."""
    rng = np.random.default_rng(Q)
    lengths = [150, 70, 9, 33, 0]
    c, raw, table = _cache(rng, lengths, [Q] * 5, 16, Hkv, D, holes=0.4)
    table[1] = -1
    c.page_table.copy_(torch.from_numpy(table))
    streams = [3, 1, 99, 0, -1, 4, 2]
    q = torch.from_numpy(rng.standard_normal((len(streams), Q, H, D))).to(DEV, torch.float16)
    out, lse = c.attend(1, q, streams=_i32(streams))
    for b, s in enumerate(streams):
        if not 0 <= s < 5 or s == 1:
            assert (out[b] == 0).all() and torch.isneginf(lse[b]).all()
            continue
        k, v, there = _tokens(raw, table, s, 1, 16, D, (0, -3))
        _check(out[b], lse[b], R.attend(q[b].double().cpu().numpy(), k, v, there, lengths[s], Q, H // Hkv, D ** -0.5, 0),
               "fp16", D)


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 3), (4, 12)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("Q", [1, 6, 70])
def test_attend_strides(offset, pad, dtype, Q):
    """Queries and outputs as slices at any element offset, heads before tokens in memory, results like the packed ones'."""
    rng = np.random.default_rng(7)
    B, H, Hkv, D, P = 3, 6, 2, 128, 16
    c, _, _ = _cache(rng, [50, 3, 200], [Q] * 3, P, Hkv, D)
    q = torch.from_numpy(rng.standard_normal((B, Q, H, D))).to(DEV, DT[dtype])
    want, want_lse = c.attend(0, q)

    def strided():
        flat = torch.full((offset + B * H * (Q * (D + pad) + pad),), 7.0, dtype=DT[dtype], device=DEV)
        return flat, flat[offset:].as_strided((B, Q, H, D), (H * (Q * (D + pad) + pad), D + pad, Q * (D + pad) + pad, 1))
    _, qs = strided()
    qs.copy_(q)
    flat, o = strided()
    got, lse = c.attend(0, qs, out=o)
    assert got is o and torch.equal(o, want) and torch.equal(lse, want_lse)
    untouched = torch.ones_like(flat, dtype=torch.bool)
    untouched[offset:].as_strided(o.shape, o.stride()).fill_(False)
    assert (flat[untouched] == 7).all()


def test_attend_extreme_queries():
    """Queries near the ends of bf16's range, of one size in a row and mixed with tiny ones; a NaN stays in its own row."""
    rng = np.random.default_rng(3)
    c, raw, table = _cache(rng, [100], [6], 16, 1, 128, k_exp=-20, v_exp=20)
    q = rng.standard_normal((1, 6, 4, 128))
    for i, e in enumerate((100, 60, -40, -110)):
        q[0, i] *= 2.0 ** e
    q[0, 4, :, ::3] *= 2.0 ** -30
    qt = torch.from_numpy(q).to(DEV, torch.bfloat16)
    qt[0, 5, 2, 7] = float("nan")
    k, v, there = _tokens(raw, table, 0, 0, 16, 128, (-20, 20))
    for scale_exp, rows in ((-86, [0]), (-46, [1]), (54, [2]), (126, [3]), (14, [4])):
        out, lse = c.attend(0, qt, scale=2.0 ** scale_exp)
        ref = R.attend(qt[0].double().cpu().numpy(), k, v, there, 100, 6, 4, 2.0 ** scale_exp, 0)
        for i in rows:
            _check(out[0, i:i + 1], lse[0, i:i + 1], [x[i:i + 1] for x in ref], "bf16", 128)
    out, lse = c.attend(0, qt, scale=2.0 ** 14)
    assert out[0, 5, 2].isnan().all() and lse[0, 5, 2].isnan()
    assert not out[0, 5, [0, 1, 3]].isnan().any()


def test_attend_nan_in_the_cache_is_seen():
    rng = np.random.default_rng(4)
    c, raw, table = _cache(rng, [40], [1], 16, 2, 64)
    k = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    k[0, 0, 1, 20] = float("nan")
    c.append(0, k, torch.zeros_like(k))
    out, lse = c.attend(0, torch.ones(1, 1, 4, 64, dtype=torch.bfloat16, device=DEV))
    assert not out[0, 0, :2].isnan().any() and out[0, 0, 2:].isnan().all() and lse[0, 0, 2:].isnan().all()


@pytest.mark.parametrize("Q", [1, 17, 64])
def test_attend_repeats_bit_for_bit_and_alone(Q):
    """The same call gives the same bits; the workspace is left as the next call needs it; another stream works as well."""
    rng = np.random.default_rng(5)
    lengths = [3000, 10, 700, 1500, 2, 0]
    c, _, _ = _cache(rng, lengths, [Q] * 6, 16, 2, 128)
    q = torch.from_numpy(rng.standard_normal((6, Q, 8, 128))).to(DEV, torch.bfloat16)
    first = c.attend(0, q)
    for _ in range(3):
        out, lse = c.attend(0, q)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = torch.zeros(S.sam_cache_attend_workspace_bytes(c.handle, 6, Q, 8), dtype=torch.uint8, device=DEV)
    side.wait_stream(torch.cuda.current_stream())
    out, lse = c.attend(0, q, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


def test_attend_in_a_graph():
    rng = np.random.default_rng(6)
    c, _, _ = _cache(rng, [900, 30], [4, 4], 16, 2, 128)
    q = torch.from_numpy(rng.standard_normal((2, 4, 8, 128))).to(DEV, torch.bfloat16)
    out, lse = c.attend(0, q)
    want = out.clone(), lse.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attend(0, q, out=out, lse=lse)
    for _ in range(3):
        out.fill_(9)
        lse.fill_(9)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


def _inputs(rng, shape, dtype):
    """Normal numbers of many sizes, exact ties of both roundings, zeros, infinities and NaN."""
    x = rng.standard_normal(shape) * 2.0 ** rng.integers(-12, 9, size=shape[:-1] + (1,))
    flat = x.reshape(-1, 16)
    flat[0] = 0
    for r, s in enumerate((1.0, 0.3125, 2.0 ** -9, 448.0)):
        flat[1 + r] = s * np.array([6, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, -.25, -.75, -1.25, -1.75, -2.5, -3.5, -5, -0.0])
    if len(flat) > 8:
        flat[5] = 2.0 ** -14 * 1.5      # below half the smallest scale
        flat[6, 3], flat[7, 9] = np.inf, np.nan
    return torch.from_numpy(x).to(DEV, DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("B,Q,Hkv,D,P,k_exp,v_exp", [(1, 1, 8, 128, 16, 0, 0), (3, 17, 2, 128, 16, 0, -3), (2, 70, 3, 64, 32, 2, -5),
                                                     (1, 700, 1, 64, 128, -1, 4), (40, 3, 4, 128, 16, 0, -24)])
def test_append_and_read(B, Q, Hkv, D, P, k_exp, v_exp, dtype):
    """Bytes and values equal the definition's; what is not named is left alone."""
    rng = np.random.default_rng(Q)
    lengths = rng.integers(0, 3 * P, size=B)
    n_new = np.maximum(rng.integers(-1, Q + 3, size=B), 0)
    n_new[0] = Q
    c, raw, table = _cache(rng, lengths, n_new, P, Hkv, D, k_exp=k_exp, v_exp=v_exp, garbage=False)
    # head before token in memory, as a projection's slice may have it
    kv = _inputs(rng, (2, B, Hkv, Q, D), dtype).permute(0, 1, 3, 2, 4)
    c.append(1, kv[0], kv[1], n_new=_i32(n_new))
    got_codes, got_scales = R.unpack_pages(c.pages.cpu().numpy(), D)
    codes, scales = R.unpack_pages(raw, D)
    x = kv.double().cpu().numpy()
    for w, exp in enumerate((k_exp, v_exp)):
        qc, qs = R.quantise(x[w], exp)
        for b in range(B):
            for i in range(min(n_new[b], Q)):
                pos = lengths[b] + i
                page = table[b, pos // P] if pos // P < table.shape[1] else -1
                if page >= 0:
                    codes[w][page, 1, :, pos % P] = qc[b, i]
                    scales[w][page, 1, :, pos % P] = qs[b, i]
    assert (got_scales == scales).all()
    assert (got_codes == codes).all()
    k, v = c.read(1, first=_i32(lengths), n=_i32(n_new), max_n=Q + 1, dtype=DT[dtype])
    for w, (t, exp) in enumerate(((k, k_exp), (v, v_exp))):
        want = np.zeros((B, Q + 1, Hkv, D))
        for b in range(B):
            for i in range(min(n_new[b], Q + 1)):
                pos = lengths[b] + i
                page = table[b, pos // P] if pos // P < table.shape[1] else -1
                if page >= 0:
                    want[b, i] = R.values(codes[w][page, 1, :, pos % P], scales[w][page, 1, :, pos % P], exp)
        with np.errstate(over="ignore"):
            want = torch.from_numpy(want).to(DT[dtype]).double().numpy()
        assert np.array_equal(t.double().cpu().numpy(), want, equal_nan=True)


def test_append_unaligned_and_named_streams():
    rng = np.random.default_rng(9)
    c, raw, table = _cache(rng, [5, 0, 20], [8] * 3, 16, 2, 64)
    flat = torch.from_numpy(rng.standard_normal(1 + 2 * 3 * 4 * 2 * 67)).to(DEV, torch.bfloat16)
    k, v = (flat[1 + w * 3 * 4 * 2 * 67:].as_strided((3, 4, 2, 64), (4 * 2 * 67, 2 * 67, 67, 1)) for w in range(2))
    c.append(0, k, v, streams=_i32([2, 7, 0]))
    rk, rv = c.read(0, first=_i32([20, 0, 5]), max_n=4, streams=_i32([2, 7, 0]))
    assert (rk[1] == 0).all() and (rv[1] == 0).all()
    for b in (0, 2):
        for x, y, exp in ((k, rk, 0), (v, rv, -3)):
            want = R.values(*R.quantise(x[b].double().cpu().numpy(), exp), exp)
            assert (y[b].double().cpu().numpy() == want).all()
    left = c.pages.cpu().numpy()
    for page in table[1][table[1] >= 0]:
        assert (left[page] == raw[page]).all()


def test_append_ignores_strides_of_single_rows():
    """Keys and values of one row and one token whose layouts differ only where there is nothing to step over."""
    c = S.SamCache(2, 16, 1, 2, 1, 2, 64, device=DEV)
    k = torch.randn(1, 1, 2, 64, device=DEV).to(torch.bfloat16)
    v = torch.randn(4, 3, 2, 64, device=DEV).to(torch.bfloat16)[2:3, 1:2]
    assert k.stride() != v.stride()
    c.reserve(_i32([1]))
    c.append(0, k, v)
    for y, x in zip(c.read(0, max_n=1), (k, v)):
        assert (y.double().cpu().numpy() == R.values(*R.quantise(x.double().cpu().numpy(), 0), 0)).all()
    with pytest.raises(ValueError):
        c.append(0, k.expand(2, 2, 2, 64), torch.zeros(2, 2, 2, 64, dtype=torch.bfloat16, device=DEV))


def test_long_offsets():
    """A pool beyond 4 GB: bytes past 2^32 are reached, read and attended to."""
    P, Hkv, D, L = 1024, 8, 128, 4
    page = S.sam_cache_page_bytes(P, L, Hkv, D)
    n_pages = (5 << 30) // page
    c = S.SamCache(n_pages, P, 2, 4, L, Hkv, D, device=DEV)
    c.page_table[0, 0], c.page_table[0, 1], c.page_table[1, 0] = n_pages - 1, n_pages - 2, 0
    c.seq_len.copy_(_i32([1020, 0]))
    rng = np.random.default_rng(11)
    kv = torch.from_numpy(rng.standard_normal((2, 2, 9, Hkv, D))).to(DEV, torch.bfloat16)
    c.pages[n_pages - 1].zero_()
    c.append(3, kv[0], kv[1])
    k, v = c.read(3, first=c.seq_len, max_n=9)
    for w, t in enumerate((k, v)):
        want = R.values(*R.quantise(kv[w].double().cpu().numpy(), 0), 0)
        assert (t.double().cpu().numpy() == want).all()
    q = torch.from_numpy(rng.standard_normal((2, 9, 8, D))).to(DEV, torch.bfloat16)
    out, lse = c.attend(3, q)
    for b, n0 in ((0, 1020), (1, 0)):
        kk, vv = (np.concatenate([np.zeros((n0, Hkv, D)), t[b].double().cpu().numpy()]) for t in (k, v))
        _check(out[b], lse[b], R.attend(q[b].double().cpu().numpy(), kk, vv, np.ones(n0 + 9, bool), n0, 9, 1, D ** -0.5, 0),
               "bf16", D)
    assert math.isfinite(float(lse.max()))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,Q,H,Hkv,P", [(128, 12, 32, 8, 16), (64, 9, 40, 8, 64), (128, 5, 32, 8, 32), (64, 2, 32, 8, 16), (128, 1, 24, 8, 128)])
def test_attend_many_steps(D, Q, H, Hkv, P, dtype):
    """Enough units for several per warp and CTA, and scores that climb along the context, so that the reference of the
    weights has to be raised again and again, and row by row at different places."""
    rng = np.random.default_rng(D + Q)
    lengths = [2600, 1900, 40, 2222]
    c, raw, table = _cache(rng, lengths, [Q] * 4, P, Hkv, D, n_layers=1)
    # the scales of the keys grow with the position: 2^-3 .. 2^3
    for s in range(4):
        for i, page in enumerate(table[s][table[s] >= 0]):
            for t in range(P // 16):
                e = min(0x50, 0x20 + 8 * ((i * P + t * 16) * 6 // 2600))
                raw[page, 0, :, t, 16 * D:17 * D] = np.minimum(raw[page, 0, :, t, 16 * D:17 * D] & 7 | e, 0x57)
    c.pages.copy_(torch.from_numpy(raw))
    q = torch.from_numpy(rng.standard_normal((4, Q, H, D)) * rng.uniform(0.05, 1.5, (4, Q, H, 1))).to(DEV, DT[dtype])
    out, lse = c.attend(0, q)
    for b in range(4):
        k, v, there = _tokens(raw, table, b, 0, P, D, (0, -3))
        _check(out[b], lse[b], R.attend(q[b].double().cpu().numpy(), k, v, there, lengths[b], Q, H // Hkv, D ** -0.5, 0), dtype, D)
    assert c.status()[1] == 0


@pytest.mark.parametrize("scale", [0.0, -0.09, 1e-30])
@pytest.mark.parametrize("Q", [1, 4, 40])
def test_attend_scales(scale, Q):
    """No scale, a negative one, and one that makes all weights alike."""
    rng = np.random.default_rng(12)
    c, raw, table = _cache(rng, [333], [Q], 16, 2, 128)
    q = torch.from_numpy(rng.standard_normal((1, Q, 8, 128))).to(DEV, torch.bfloat16)
    out, lse = c.attend(1, q, scale=scale)
    k, v, there = _tokens(raw, table, 0, 1, 16, 128, (0, -3))
    _check(out[0], lse[0], R.attend(q[0].double().cpu().numpy(), k, v, there, 333, Q, 4, scale, 0), "bf16", 128)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Q,H", [(6, 1), (6, 4), (6, 8)])
def test_nan_reaches_only_the_rows_that_see_it(Q, H, D):
    """A NaN among the values of a token: earlier rows, and rows whose window has passed it, do not know of it; the others have it
    in its 16 channels only.  Among the keys: the rows that see it are NaN, the others are not."""
    window = 4
    rng = np.random.default_rng(13)
    for where in ("value", "key"):
        c, _, _ = _cache(rng, [70], [Q], 16, 1, D, n_layers=1)
        kv = torch.from_numpy(rng.standard_normal((2, 1, Q, 1, D))).to(DEV, torch.bfloat16)
        kv[1 if where == "value" else 0, 0, 1, 0, 37] = float("nan")
        c.append(0, kv[0], kv[1])
        q = torch.from_numpy(rng.standard_normal((1, Q, H, D))).to(DEV, torch.bfloat16)
        for win, seen in ((0, range(1, Q)), (window, range(1, 1 + window))):
            out, lse = c.attend(0, q, window=win)
            nan = out[0].isnan()
            for i in range(Q):
                want = torch.zeros(H, D, dtype=torch.bool, device=DEV)
                if i in seen:
                    want[:, 32:48] = True
                    if where == "key":
                        want[:] = True
                assert torch.equal(nan[i], want), (where, win, i)
                assert bool(lse[0, i].isnan().all()) == (where == "key" and i in seen)


def test_attend_refuses_what_does_not_fit():
    c = S.SamCache(4, 16, 2, 2, 1, 2, 64, device=DEV)
    q = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16, device=DEV)
    i32 = torch.zeros(2, dtype=torch.int32, device=DEV)
    for bad in (q.float(), q[..., :32], q[0], q.transpose(2, 3), q.cpu()):
        with pytest.raises(ValueError):
            c.attend(0, bad)
    for kw in (dict(out=q.half()), dict(out=q[:1]), dict(lse=torch.zeros(2, 1, 4, device=DEV).half()), dict(n_new=i32[:1]),
               dict(streams=i32.long())):
        with pytest.raises(ValueError):
            c.attend(0, q, **kw)
    with pytest.raises(S.SamError) as e:
        c.attend(1, q)
    assert e.value.status == -1
    with pytest.raises(S.SamError):
        c.attend(0, q[:, :, :3])                       # three query heads over two key heads
    with pytest.raises(S.SamError) as e:
        c.attend(0, q, workspace=torch.zeros(512, dtype=torch.uint8, device=DEV))
    assert e.value.status == -5
    k = torch.zeros(2, 1, 2, 64, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError):
        c.append(0, k, k.half())
    with pytest.raises(ValueError):
        c.append(0, k[:, :, :1], k[:, :, :1])
    with pytest.raises(ValueError):
        c.append(0, k, k.expand(2, 1, 2, 64).transpose(0, 1).contiguous().transpose(0, 1), n_new=i32.float())
    with pytest.raises(ValueError):
        c.read(0, out=(k, k.half()))
    with pytest.raises(ValueError):
        S.SamCache(4, 16, 2, 2, 1, 2, 64, device=DEV, tensors=dict(seq_len=i32.long()))
