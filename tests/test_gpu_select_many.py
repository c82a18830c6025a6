"""Selections with so many lists that a warp takes each: more than eight lists and heads for every multiprocessor."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from tests.test_gpu_cache_attend import DEV, DT, _cache, _i32
from tests.test_gpu_select import _bounds, _query_codes

pytestmark = pytest.mark.gpu


def _lists(q, length, n_new, table, codes, exps, P, n_sink, n_recent, n_blocks, layer):
    """q [Q, Hkv, D] in 64 bits, one token a list -> [Q, Hkv, n_blocks]: the definition, a matrix of scores at a time."""
    Q, Hkv, D = q.shape
    out = -np.ones((Q, Hkv, n_blocks), np.int32)
    there = np.flatnonzero(table >= 0)
    for h in range(Hkv):
        hi, lo = (codes[table[there], layer, h, k].astype(np.int64) for k in range(2))
        e_k = exps[table[there], layer, h].astype(np.int64)
        for i in range(min(n_new, Q)):
            w, e_q = _query_codes(q[i, h])
            score = (np.maximum(w, 0) @ hi.T + np.minimum(w, 0) @ lo.T).astype(np.float32) * np.float32(2.0 ** e_q) * np.exp2(e_k).astype(np.float32)
            p = length + i
            up = there <= p // P
            first = (there < n_sink) | (there > p // P - n_recent)
            rank = np.where(first, 0, np.where(e_k == 127, 1, 2))
            order = np.lexsort((there, np.where(rank == 2, -score, 0.0), rank))
            keep = np.sort(there[order[up[order]][:n_blocks]])
            out[i, h, :len(keep)] = keep
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("max_len,kernel", [(3000, "512 pages"), (9000, "1024 pages")])
def test_a_warp_a_list(max_len, kernel, dtype):
    """Ties, holes, pages with NaN, queries of zero; short contexts beside long ones; rows with fewer tokens than the rest."""
    rng = np.random.default_rng(max_len)
    Q, Hkv, D, P = 160, 4, 64, 16
    lengths, n_new = [max_len, 100, max_len - 500], [Q, Q, Q - 7]
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert len(lengths) * Q * Hkv > 8 * sms
    c, raw, table = _cache(rng, lengths, [Q] * 3, P, Hkv, D, holes=0.1, garbage=False)
    assert (table.shape[1] <= 512) == (kernel == "512 pages") and table.shape[1] <= 1024
    raw[..., 16 * D:17 * D] = rng.integers(0x28, 0x40, size=raw[..., 16 * D:17 * D].shape)
    held = table[0][table[0] >= 0]
    raw[held[20:80]] = raw[held[np.arange(60) % 5]]                         # whole classes tie
    raw[held[[33, 90]], 1, 2, 0, 16 * D] = 0x7f                             # NaN among the keys
    c.pages.copy_(torch.from_numpy(raw))
    b = S.SamBounds(c)
    b.rebuild()
    q = torch.from_numpy(rng.standard_normal((3, Q, Hkv, D)))
    q[:, 3::17] = 0.0
    q = q.to(DEV, DT[dtype])
    codes, exps = _bounds(raw, D, 0)
    x = q.double().cpu().numpy()
    for n_sink, n_recent, n_blocks in ((1, 2, 3), (1, 2, 24), (0, 1, 150)):
        got = b.select(1, q, n_blocks, n_sink=n_sink, n_recent=n_recent, n_new=_i32(n_new)).cpu().numpy()
        for r in range(3):
            want = _lists(x[r], lengths[r], n_new[r], table[r], codes, exps, P, n_sink, n_recent, n_blocks, 1)
            assert (got[r] == want).all(), (n_blocks, r)
