"""Queries and keys turned on their way into the cache, against 64-bit (angles: 80-bit) numpy."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from tests import cache_reference as R
from tests.test_gpu_cache_attend import BITS, DEV, DT, _i32

pytestmark = pytest.mark.gpu


def _empty_cache(lengths, Q, P, Hkv, D, n_layers=2, k_exp=0, v_exp=-3, spare=2):
    held = [-(-(l + Q) // P) for l in lengths]
    c = S.SamCache(sum(held) + spare, P, len(lengths), max(held), n_layers, Hkv, D, k_exp, v_exp, device=DEV)
    table = -np.ones((len(lengths), max(held)), np.int32)
    order, at = np.random.default_rng(1).permutation(sum(held) + spare), 0
    for s, n in enumerate(held):
        table[s, :n] = order[at:at + n]
        at += n
    c.page_table.copy_(torch.from_numpy(table))
    c.seq_len.copy_(_i32(lengths))
    c.pages.zero_()
    return c, table


def _turn(x, pos, f, interleaved, factor):
    """x [Q, H, D] in 64 bits turned to pos [Q], and |a| + |b| of each channel's pair (0 where nothing is turned)."""
    R2 = len(f)
    angle = np.asarray(pos, np.longdouble)[:, None] * np.asarray(f, np.longdouble)
    cos, sin = (np.asarray(g(angle), np.float64)[:, None] * factor for g in (np.cos, np.sin))
    a, b = (slice(0, 2 * R2, 2), slice(1, 2 * R2, 2)) if interleaved else (slice(0, R2), slice(R2, 2 * R2))
    y, size = x.copy(), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., b] * cos + x[..., a] * sin
    size[..., a] = size[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * abs(factor)
    return y, size


# A turned channel before it is rounded: the angle is off by pi 2^-25 (a half turn's fraction as a float) and pi 2^-31, sine
# and cosine by two units in the last place (2^-23 each at most), their product with the factor, the two products and the sum by 2^-24 each:
# less than 2^-20.9 of |a| + |b| in all.
ROTATION = 2.0 ** -20.9


def _check_queries(got, x, size, dtype):
    got = got.double().cpu().numpy()
    off = ROTATION * size
    e = np.floor(np.log2(np.abs(x) + off + 1e-300))
    bound = off + np.where(size > 0, np.maximum(2.0 ** (e - BITS[dtype]), 2.0 ** -25 if dtype == "fp16" else 2.0 ** -134), 0)
    assert (np.abs(got - x) <= bound).all()


def _check_codes(codes, scales, x, size, exp):
    """codes [.., D], scales [.., D/16]: the scale is that of some values within reach, and each code the nearest for one."""
    off = ROTATION * size
    b, o = (t.reshape(*x.shape[:-1], -1, 16) for t in (np.abs(x), off))
    lo, hi = (R.nearest(R.E4M3, np.minimum(t / (6 * 2.0 ** exp), 448.0)) for t in ((b - o).max(-1).clip(0) * (1 - 2e-7), (b + o).max(-1) * (1 + 2e-7)))
    assert ((scales >= lo) & (scales <= hi)).all()
    v = R.values(codes, scales, exp)
    s = np.repeat(R.E4M3[scales], 16, -1) * 2.0 ** exp
    grid = np.concatenate([R.E2M1, -R.E2M1])
    best = np.abs(grid * s[..., None] - x[..., None]).min(-1)
    slack = 2 * off + 2.0 ** -21 * np.abs(x)               # the quotient is rounded to 22 bits
    assert (np.abs(v - x) <= best + slack).all()


CASES = [
    # lengths, n_new, Q, H, Hkv, D, P, rotary, interleaved, factor
    ([0], [1], 1, 1, 1, 64, 16, 64, False, 1.0),
    ([0, 1, 15, 16, 17], [1] * 5, 1, 8, 2, 128, 16, 128, False, 1.0),
    ([5, 0, 100, 33], [0, 3, 5, -2], 5, 6, 2, 128, 16, 128, True, 1.0),
    ([63, 64, 65], [2, 1, 2], 2, 7, 1, 64, 64, 32, False, 0.7),
    ([300, 31], [17, 4], 17, 8, 2, 128, 32, 96, False, 1.2),
    ([300, 31], [17, 17], 17, 28, 4, 128, 32, 64, True, -1.0),
    ([1 << 20], [40], 40, 5, 5, 64, 1024, 64, False, 1.0),
    ([211], [700], 700, 2, 1, 128, 32, 32, True, 1.0),
    ([3], [9], 9, 0, 2, 128, 16, 128, False, 1.0),
    ([40] * 300, [9] * 300, 9, 2, 1, 64, 16, 32, False, 1.0),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append_rotated(case, dtype):
    lengths, n_new, Q, H, Hkv, D, P, rot, inter, factor = CASES[case]
    rng = np.random.default_rng(case)
    B = len(lengths)
    c, table = _empty_cache(lengths, Q, P, Hkv, D)
    f = 10000.0 ** (-np.arange(rot // 2) * 2 / rot)
    rope = S.SamRope(f, interleaved=inter, factor=factor, device=DEV)
    qkv = torch.from_numpy(rng.standard_normal((B, Q, H + 2 * Hkv, D))).to(DEV, DT[dtype])
    q, k, v = qkv.split([H, Hkv, Hkv], 2)
    out = torch.full((B, Q, H, D), 7.0, dtype=DT[dtype], device=DEV)
    assert c.append_rotated(1, q, k, v, rope, n_new=_i32(n_new), out=out) is out
    plain, _ = _empty_cache(lengths, Q, P, Hkv, D)
    plain.append(1, k, v, n_new=_i32(n_new))
    raw, want = c.pages.cpu().numpy(), plain.pages.cpu().numpy()
    # values, and the blocks of 16 channels that are not turned, are what the plain append stores; nothing else is touched
    assert (raw[..., 8 * D:16 * D] == want[..., 8 * D:16 * D]).all() and (raw[..., 17 * D:] == want[..., 17 * D:]).all()
    codes, scales = R.unpack_pages(raw, D)
    codes2, scales2 = R.unpack_pages(want, D)
    assert (codes[0][..., rot:] == codes2[0][..., rot:]).all() and (scales[0][..., rot // 16:] == scales2[0][..., rot // 16:]).all()
    assert not raw[:, 0].any()
    for b in range(B):
        n = max(n_new[b], 0)
        assert (out[b, n:] == 0).all()
        if n == 0:
            continue
        pos = lengths[b] + np.arange(n)
        y, size = _turn(q[b, :n].double().cpu().numpy(), pos, f, inter, factor)
        _check_queries(out[b, :n], y, size, dtype)
        y, size = _turn(k[b, :n].double().cpu().numpy(), pos, f, inter, factor)
        page, slot = table[b, pos // P], pos % P
        _check_codes(codes[0][page, 1, :, slot], scales[0][page, 1, :, slot], y, size, 0)
    touched = np.zeros(raw.shape[0] * P, bool)
    for b in range(B):
        pos = lengths[b] + np.arange(max(n_new[b], 0))
        touched[table[b, pos // P] * P + pos % P] = True
    assert not codes[0][:, 1].transpose(0, 2, 1, 3).reshape(-1, Hkv * D)[~touched].any()


@pytest.mark.parametrize("positions", [[0, 1, 7, 250_000, (1 << 30) - 1, (1 << 31) - 1, -1, -(1 << 31)]])
@pytest.mark.parametrize("f", [1.0, 0.31831, 3e-5, 2.7])
def test_far_positions(positions, f):
    """The angle is exact to a fraction of a turn at any position, given explicitly."""
    Q = len(positions)
    c, _ = _empty_cache([0], Q, 16, 1, 64)
    rope = S.SamRope(np.full(16, f), device=DEV)
    rng = np.random.default_rng(0)
    q = torch.from_numpy(rng.standard_normal((1, Q, 3, 64))).to(DEV, torch.float16)
    k = torch.zeros(1, Q, 1, 64, dtype=torch.float16, device=DEV)
    got = c.append_rotated(0, q, k, k, rope, positions=_i32([positions]))
    y, size = _turn(q[0].double().cpu().numpy(), positions, np.full(16, f), False, 1.0)
    # the turns of a position have 64 bits, of which 2^31 positions leave 33: 2^-32 of a turn more
    size = size * (1 + 2 * np.pi * 2.0 ** -32 / ROTATION)
    _check_queries(got[0], y, size, "fp16")


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 3), (4, 12)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("inter", [False, True])
def test_strides_and_in_place(offset, pad, dtype, inter):
    rng = np.random.default_rng(5)
    B, Q, H, Hkv, D = 3, 5, 6, 2, 128
    rope = S.SamRope(0.9 ** np.arange(64), interleaved=inter, device=DEV)
    q = torch.from_numpy(rng.standard_normal((B, Q, H, D))).to(DEV, DT[dtype])
    k, v = (torch.from_numpy(rng.standard_normal((B, Q, Hkv, D))).to(DEV, DT[dtype]) for _ in range(2))
    c, _ = _empty_cache([50, 3, 200], Q, 16, Hkv, D)
    want = c.append_rotated(0, q, k, v, rope)

    def strided(x):
        heads = x.shape[2]
        flat = torch.full((offset + B * heads * (Q * (D + pad) + pad),), 7.0, dtype=x.dtype, device=DEV)
        y = flat[offset:].as_strided(x.shape, (heads * (Q * (D + pad) + pad), D + pad, Q * (D + pad) + pad, 1))
        y.copy_(x)
        return flat, y
    flat, qs = strided(q)
    c2, _ = _empty_cache([50, 3, 200], Q, 16, Hkv, D)
    got = c2.append_rotated(0, qs, strided(k)[1], strided(v)[1], rope, out=qs)
    assert got is qs and torch.equal(qs, want) and torch.equal(c.pages, c2.pages)
    untouched = torch.ones_like(flat, dtype=torch.bool)
    untouched[offset:].as_strided(qs.shape, qs.stride()).fill_(False)
    assert (flat[untouched] == 7).all()


def test_named_streams_absent_pages_and_the_end_of_the_table():
    """Unknown streams leave nothing and read as zero; positions without a page, or behind the table, are left out while
    their queries are turned."""
    rng = np.random.default_rng(2)
    c, table = _empty_cache([20, 40, 0], 16, 16, 1, 64)
    table[1, 3] = -1
    c.page_table.copy_(torch.from_numpy(table))
    f = 0.5 ** np.arange(32)
    rope = S.SamRope(f, device=DEV)
    streams = [1, 7, 0, -1]
    q, k = (torch.from_numpy(rng.standard_normal((4, 30, 1, 64))).to(DEV, torch.bfloat16) for _ in range(2))
    got = c.append_rotated(0, q, k, k, rope, streams=_i32(streams))
    assert (got[1] == 0).all() and (got[3] == 0).all()
    codes, _ = R.unpack_pages(c.pages.cpu().numpy(), 64)
    for b, s in ((0, 1), (2, 0)):
        start = [20, 40, 0][s]
        y, size = _turn(q[b].double().cpu().numpy(), start + np.arange(30), f, False, 1.0)
        _check_queries(got[b], y, size, "bf16")
        for i in range(start, min(start + 30, table.shape[1] * 16)):
            page = table[s, i // 16]
            assert page < 0 or codes[0][page, 0, :, i % 16].any()
    held = table[[0, 1]][table[[0, 1]] >= 0]
    assert not codes[0][np.setdiff1d(np.arange(codes[0].shape[0]), held)].any()


def test_nan_and_infinity_stay_in_their_blocks():
    c, table = _empty_cache([0], 4, 16, 1, 128)
    rope = S.SamRope(np.full(32, 0.3), device=DEV)                # channels 0 .. 31 with 32 .. 63
    k = torch.ones(1, 4, 1, 128, dtype=torch.bfloat16, device=DEV)
    k[0, 1, 0, 5] = float("nan")
    k[0, 2, 0, 100] = float("inf")
    q = k.clone()
    out = c.append_rotated(0, q, k, k.clone(), rope)
    kk, vv = c.read(0, first=_i32([0]), n=_i32([4]), max_n=4)
    kk, vv = kk[0, :, 0].float(), vv[0, :, 0].float()
    assert kk[1, :16].isnan().all() and kk[1, 32:48].isnan().all() and not kk[1, 16:32].isnan().any() and not kk[1, 48:].isnan().any()
    assert kk[2, 100] == 6 * 448 and (kk[2, 96:100] == 0).all() and (kk[3] != 0).all()
    assert vv[1, :16].isnan().all() and not vv[1, 16:].isnan().any() and vv[2, 100] == 6 * 448 / 8
    assert out[0, 1, 0].isnan().nonzero().flatten().tolist() == [5, 37] and out[0, 2, 0].isinf().nonzero().flatten().tolist() == [100]
