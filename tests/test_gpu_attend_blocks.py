"""Attention over listed blocks against 64-bit numpy, with the bounds of the dense attention's tests."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from tests import cache_reference as R
from tests.test_gpu_cache_attend import DEV, DT, _cache, _check, _i32, _tokens

pytestmark = pytest.mark.gpu


def _lists(rng, lengths, n_new, Q, Hkv, P, share, n_blocks, max_pages):
    """Ascending lists of different blocks up to the run's last, its own among them."""
    out = -np.ones((len(lengths), -(-Q // share), Hkv, n_blocks), np.int32)
    for b, (t, n) in enumerate(zip(lengths, n_new)):
        for l in range(out.shape[1]):
            last = min((t + min((l + 1) * share, max(n, l * share + 1)) - 1) // P, max_pages - 1)
            own = list(range(max(0, min((t + l * share) // P, last)), last + 1))[-n_blocks:]
            for h in range(Hkv):
                rest = rng.permutation(own[0])[:n_blocks - len(own)] if own[0] else []
                x = sorted(set(own) | set(int(i) for i in rest))
                out[b, l, h, :len(x)] = x
    return out


def _compare(c, raw, table, q, blocks, out, lse, lengths, n_new, P, share, scale, dtype, layer, rows=None):
    Q, H, D = q.shape[1:]
    Hkv = raw.shape[2]
    g = H // Hkv
    for b in range(q.shape[0]):
        s = b if rows is None else rows[b]
        if not 0 <= s < len(lengths):
            assert (out[b] == 0).all() and torch.isneginf(lse[b]).all()
            continue
        k, v, there = _tokens(raw, table, s, layer, P, D, (0, -3))
        for l in range(blocks.shape[1]):
            i0, i1 = l * share, min((l + 1) * share, Q)
            n = min(max(n_new[b] - i0, 0), i1 - i0)
            for h in range(Hkv):
                heads = slice(h * g, (h + 1) * g)
                used = blocks[b, l, h, :(lengths[s] + i0 + max(n, 1) - 1) // P + 1]
                on = np.zeros(len(there), bool)
                for i in used:
                    if 0 <= i < table.shape[1]:
                        on[i * P:(i + 1) * P] = there[i * P:(i + 1) * P]
                ref = R.attend(q[b, i0:i1, heads].double().cpu().numpy(), k[:, h:h + 1], v[:, h:h + 1], on, lengths[s] + i0, n, g, scale, 0)
                # Weights are fp16 against a reference that lies at least 4 (in powers of two) below the largest score: their sum is 2^4 or more, and
                # one that is subnormal is off by up to 2^-25, 2^-29 of the sum.  As a part of the 2^-11 that _check allows of the mean of |v|:
                seen = on & (np.arange(len(on)) < lengths[s] + i0 + n) & (n > 0)
                ref = (*ref[:2], ref[2] + 2.0 ** -18 * np.abs(v[seen, h]).sum(0), ref[3])
                assert np.isfinite(ref[2]).all()
                _check(out[b, i0:i1, heads], lse[b, i0:i1, heads], ref, dtype, D)


CASES = [
    # lengths, n_new, Q, H, Hkv, D, P, share, n_blocks
    ([0], [1], 1, 1, 1, 64, 16, 1, 1),
    ([0, 1, 15, 16, 17, 200], [1] * 6, 1, 8, 2, 128, 16, 1, 4),
    ([333, 1000], [1, 1], 1, 32, 8, 128, 16, 1, 7),
    ([5, 0, 100, 33], [0, 3, 5, -2], 5, 6, 2, 128, 16, 1, 3),
    ([5, 0, 100, 333], [0, 3, 5, 2], 5, 6, 2, 64, 16, 2, 5),
    ([63, 64, 65, 127, 700], [2, 1, 2, 1, 2], 2, 7, 1, 64, 64, 2, 3),
    ([300, 31], [17, 4], 17, 8, 2, 128, 32, 17, 6),
    ([900, 31], [17, 17], 17, 8, 1, 128, 16, 17, 40),
    ([700], [33], 33, 10, 2, 128, 16, 8, 9),
    ([900], [50], 50, 28, 4, 64, 64, 16, 5),
    ([600, 5], [40, 40], 40, 16, 1, 128, 16, 40, 12),           # 640 query rows a list
    ([600], [129], 129, 2, 2, 128, 128, 129, 4),
    ([5000], [1], 1, 3, 1, 64, 1024, 1, 3),
    ([4000], [3], 3, 64, 8, 128, 16, 3, 200),
    ([0], [300], 300, 4, 2, 128, 16, 16, 6),
    ([40] * 300, [2] * 300, 2, 2, 1, 64, 16, 1, 3),              # more runs than a block has threads
    ([600, 90, 333], [17, 9, 16], 17, 16, 2, 128, 16, 17, 12),   # 136 query rows a list, and fewer
    ([300, 50], [65, 64], 65, 2, 1, 64, 16, 65, 9),              # 130
    ([100, 900], [90, 11], 90, 3, 1, 128, 32, 90, 14),           # 270
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attend_blocks(case, dtype):
    lengths, n_new, Q, H, Hkv, D, P, share, n_blocks = CASES[case]
    rng = np.random.default_rng(200 + case)
    c, raw, table = _cache(rng, lengths, [max(n, 0) for n in n_new], P, Hkv, D)
    q = torch.from_numpy(rng.standard_normal((len(lengths), Q, H, D))).to(DEV, DT[dtype])
    blocks = _lists(rng, lengths, n_new, Q, Hkv, P, share, n_blocks, table.shape[1])
    for layer, scale in ((0, None), (1, -0.31)):
        out, lse = c.attend_blocks(layer, q, _i32(blocks), share=share, n_new=_i32(n_new), scale=scale)
        _compare(c, raw, table, q, blocks, out, lse, lengths, n_new, P, share, D ** -0.5 if scale is None else scale, dtype, layer)
    assert c.status()[1] == 0


@pytest.mark.parametrize("Q,share,H", [(1, 1, 8), (9, 3, 8), (20, 20, 16)])
@pytest.mark.parametrize("P", [16, 32])
def test_any_list_will_do(Q, share, H, P):
    """Entries out of range, absent pages, blocks behind the run, in any order; rows that name their streams; lists that leave nothing."""
    rng = np.random.default_rng(Q)
    lengths = [400, 70, 9, 133, 0]
    c, raw, table = _cache(rng, lengths, [Q] * 5, P, 2, 128, holes=0.25)
    streams = [3, 1, 99, 0, -1, 4, 2]
    q = torch.from_numpy(rng.standard_normal((len(streams), Q, H, 128))).to(DEV, torch.float16)
    blocks = -np.ones((len(streams), -(-Q // share), 2, 30), np.int32)
    for at in np.ndindex(blocks.shape[:3]):
        x = rng.permutation(np.concatenate([np.arange(table.shape[1] + 4), [-1, -7, 1 << 30, -(1 << 31), (1 << 31) - 1]]))[:30]
        blocks[at][:len(x)] = x
    blocks[0, 0, 1] = -1
    out, lse = c.attend_blocks(1, q, _i32(blocks), share=share, streams=_i32(streams))
    _compare(c, raw, table, q, blocks, out, lse, lengths, [Q] * len(streams), P, share, 128 ** -0.5, "fp16", 1, streams)


@pytest.mark.parametrize("Q,share", [(1, 1), (24, 24)])
def test_a_block_twice_counts_twice(Q, share):
    rng = np.random.default_rng(3)
    c, raw, table = _cache(rng, [100], [Q], 16, 1, 128)
    q = torch.from_numpy(rng.standard_normal((1, Q, 8, 128))).to(DEV, torch.bfloat16)
    _, one = c.attend_blocks(0, q, _i32([[[[2, 3]]]]), share=share)
    out, two = c.attend_blocks(0, q, _i32([[[[2, 3, 2, 3]]]]), share=share)
    single, _ = c.attend_blocks(0, q, _i32([[[[2, 3]]]]), share=share)
    assert torch.allclose(two, one + np.log(2), atol=1e-5) and (out.float() - single.float()).abs().max() <= 2 * 2.0 ** -8 * single.float().abs().max()


@pytest.mark.parametrize("Q,H", [(1, 4), (3, 8), (17, 8), (40, 4)])
@pytest.mark.parametrize("P", [16, 64])
def test_all_blocks_are_the_dense_attention(Q, H, P):
    """With every block listed the sums are those of the dense kernel in other groups: within two roundings of one another."""
    rng = np.random.default_rng(9)
    lengths = [500, 37]
    c, _, table = _cache(rng, lengths, [Q] * 2, P, 2, 128)
    q = torch.from_numpy(rng.standard_normal((2, Q, H, 128))).to(DEV, torch.float16)
    M = table.shape[1]
    blocks = _i32(np.broadcast_to(np.arange(M), (2, 1, 2, M)))
    out, lse = c.attend_blocks(0, q, blocks, share=Q)
    want, want_lse = c.attend(0, q)
    assert (lse - want_lse).abs().max() < 1e-5
    assert ((out - want).abs().float() <= 2.0 ** -9 * want.abs().float() + 2.0 ** -10).all()


def test_nan_is_seen_by_those_who_see_it():
    """NaN among keys and values: only rows whose list and position reach it, for values only its channels."""
    rng = np.random.default_rng(4)
    for Q, share, H in ((1, 1, 4), (40, 40, 4), (6, 3, 2)):
        c, raw, table = _cache(rng, [70], [Q], 16, 1, 128, garbage=False)
        for block, part in ((1, 17 * 128 + 5 * 8 + 2), (2, 16 * 128 + 5 * 8 + 2)):      # token 5: values of block 1, keys of block 2
            raw[table[0, block], :, :, 0, part] = 0x7f
        raw[table[0, 4], :, :, 0, 17 * 128 + 8 * 8 + 1] = 0xff                          # position 72, channels 16 .. 31
        c.pages.copy_(torch.from_numpy(raw))
        q = torch.from_numpy(rng.standard_normal((1, Q, H, 128))).to(DEV, torch.bfloat16)
        lists = -(-Q // share)
        for used, keys, values in (([0, 3], False, False), ([0, 1], False, True), ([0, 2, 3], True, False), ([0, 4], False, False)):
            blocks = np.full((1, lists, 1, 3), -1, np.int32)
            blocks[..., :len(used)] = used
            out, lse = c.attend_blocks(0, q, _i32(blocks), share=share)
            nan = out[0].isnan()
            for i in range(Q):
                if keys:
                    assert nan[i].all() and lse[0, i].isnan().all()
                    continue
                want = torch.zeros(128, dtype=torch.bool, device=DEV)
                if values:
                    want[32:48] = True
                if 4 in used and 70 + i >= 72:
                    want[16:32] = True
                assert (nan[i] == want).all() and not lse[0, i].isnan().any()


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 3)])
@pytest.mark.parametrize("Q,share", [(1, 1), (6, 2), (40, 40)])
def test_strides(offset, pad, Q, share):
    rng = np.random.default_rng(7)
    B, H, Hkv, D, P = 3, 6, 2, 128, 16
    lengths = [50, 3, 200]
    c, _, table = _cache(rng, lengths, [Q] * 3, P, Hkv, D)
    q = torch.from_numpy(rng.standard_normal((B, Q, H, D))).to(DEV, torch.bfloat16)
    blocks = _i32(_lists(rng, lengths, [Q] * 3, Q, Hkv, P, share, 6, table.shape[1]))
    want, want_lse = c.attend_blocks(0, q, blocks, share=share)

    def strided():
        flat = torch.full((offset + B * H * (Q * (D + pad) + pad),), 7.0, dtype=q.dtype, device=DEV)
        return flat, flat[offset:].as_strided((B, Q, H, D), (H * (Q * (D + pad) + pad), D + pad, Q * (D + pad) + pad, 1))
    _, qs = strided()
    qs.copy_(q)
    flat, o = strided()
    got, lse = c.attend_blocks(0, qs, blocks, share=share, out=o)
    assert got is o and torch.equal(o, want) and torch.equal(lse, want_lse)
    untouched = torch.ones_like(flat, dtype=torch.bool)
    untouched[offset:].as_strided(o.shape, o.stride()).fill_(False)
    assert (flat[untouched] == 7).all()


def test_a_batch_of_uneven_lists():
    """Many streams of very different lengths, short and full lists, in one call."""
    rng = np.random.default_rng(11)
    lengths = [int(x) for x in rng.integers(0, 3000, size=40)]
    n_new = [int(x) for x in rng.integers(0, 18, size=40)]
    c, raw, table = _cache(rng, lengths, n_new, 16, 2, 128)
    q = torch.from_numpy(rng.standard_normal((40, 17, 8, 128))).to(DEV, torch.bfloat16)
    for share in (1, 17):
        blocks = _lists(rng, lengths, n_new, 17, 2, 16, share, 24, table.shape[1])
        out, lse = c.attend_blocks(0, q, _i32(blocks), share=share, n_new=_i32(n_new))
        _compare(c, raw, table, q, blocks, out, lse, lengths, n_new, 16, share, 128 ** -0.5, "bf16", 0)
