"""Attention over batches as large as the configurations that the drafts run with: work is numbered in several rounds of a CTA's
threads there (more than 256 rows in the streaming kernel, more than 896 row tiles in the wide one)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests.test_gpu_cache_attend import DEV, DT, _cache, _check, _i32
import paper_2512_18337_b200 as S

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Q,H,Hkv,D,P,longest,dtype", [
    (257, 1, 4, 2, 64, 16, 90, "bf16"), (300, 1, 2, 1, 128, 16, 90, "fp16"), (1024, 3, 1, 1, 64, 32, 60, "bf16"),
    (4096, 1, 1, 1, 64, 16, 30, "fp16"), (897, 33, 1, 1, 64, 16, 20, "bf16"), (300, 40, 8, 1, 64, 16, 20, "fp16"),
    (950, 35, 1, 1, 128, 16, 20, "bf16")])
def test_large_batches(B, Q, H, Hkv, D, P, longest, dtype):
    """Rows without new tokens, without a context and with both, and one long context among the short ones."""
    rng = np.random.default_rng(B + Q)
    lengths = rng.integers(0, longest, size=B)
    lengths[B // 2] = 5000
    lengths[[0, B - 1]] = 0, longest
    n_new = np.where(rng.random(B) < 0.2, 0, rng.integers(1, Q + 1, size=B))
    n_new[[0, B // 2, B - 1]] = 1, 1, Q
    c, raw, table = _cache(rng, lengths.tolist(), [Q] * B, P, Hkv, D, n_layers=1)
    q = torch.from_numpy(rng.standard_normal((B, Q, H, D))).to(DEV, DT[dtype])
    order = rng.permutation(B)                             # row b is stream order[b]
    out, lse = c.attend(0, q, n_new=_i32(n_new[order]), streams=_i32(order))
    assert c.status()[1] == 0
    codes, scales = R.unpack_pages(raw, D)
    kv = [R.values(codes[w], scales[w], e)[:, 0].transpose(0, 2, 1, 3) for w, e in ((0, 0), (1, -3))]     # [pages, P, Hkv, D]
    out64, lse64, q64 = out.double().cpu(), lse.double().cpu(), q.double().cpu().numpy()
    refs = []
    for b in range(B):
        s = order[b]
        pages = table[s][:-(-(lengths[s] + n_new[s]) // P)]
        k, v = (x[pages].reshape(-1, Hkv, D) for x in kv)
        refs.append(R.attend(q64[b], k, v, np.ones(len(k), bool), int(lengths[s]), int(n_new[s]), H // Hkv, D ** -0.5, 0))
    _check(out64, lse64, [np.stack(x) for x in zip(*refs)], dtype, D)


def test_more_rows_than_a_call_takes_are_refused():
    c = S.SamCache(4, 16, 5000, 1, 1, 1, 64, device=DEV)
    with pytest.raises(S.SamError) as e:
        c.attend(0, torch.zeros(4097, 1, 1, 64, dtype=torch.bfloat16, device=DEV))
    assert e.value.status == -6
