"""The wide attention kernel where the threads of a warp take different ways: query rows that end inside a warp, contexts that
several CTAs hold, NaN that only some rows see, and unaligned queries and results.  Results are the single streams' own."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests.test_gpu_cache_attend import DEV, DT, _cache, _check, _i32, _tokens

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("D,Q,H,Hkv", [(128, 33, 2, 2), (64, 45, 3, 1), (128, 129, 1, 1), (64, 11, 7, 1)])
def test_rows_that_end_inside_a_warp(D, Q, H, Hkv, offset, dtype):
    rng = np.random.default_rng(Q)
    lengths, n_new = [900, 20, 333], [Q, Q - 2, Q - 1]
    c, raw, table = _cache(rng, lengths, [Q] * 3, 16, Hkv, D, n_layers=1)
    flat = torch.from_numpy(rng.standard_normal(3 * Q * H * (D + 8) + 8)).to(DEV, DT[dtype])
    q = flat[offset:offset + 3 * Q * H * (D + 8)].view(3, Q, H, D + 8)[..., :D]
    out = torch.full_like(flat, 5)[offset:offset + 3 * Q * H * (D + 8)].view(3, Q, H, D + 8)[..., :D]
    _, lse = c.attend(0, q, n_new=_i32(n_new), out=out)
    for b in range(3):
        k, v, there = _tokens(raw, table, b, 0, 16, D, (0, -3))
        _check(out[b], lse[b], R.attend(q[b].double().cpu().numpy(), k, v, there, lengths[b], n_new[b], H // Hkv, D ** -0.5, 0), dtype, D)
    assert c.status()[1] == 0


@pytest.mark.parametrize("D,Q,H", [(128, 45, 1), (64, 45, 3), (128, 70, 2)])
@pytest.mark.parametrize("length", [70, 1500])
def test_nan_that_some_rows_of_a_warp_see(D, Q, H, length):
    """NaN values at three of the new tokens: each row has NaN in exactly the blocks of the tokens that it sees."""
    rng = np.random.default_rng(D + Q)
    c, _, _ = _cache(rng, [length], [Q], 16, 1, D, n_layers=1)
    kv = torch.from_numpy(rng.standard_normal((2, 1, Q, 1, D))).to(DEV, torch.bfloat16)
    at = {3: 5, Q // 2: 20, Q - 2: D - 1}                  # token -> channel
    for t, ch in at.items():
        kv[1, 0, t, 0, ch] = float("nan")
    c.append(0, kv[0], kv[1])
    q = torch.from_numpy(rng.standard_normal((1, Q, H, D))).to(DEV, torch.bfloat16)
    for window in (0, Q // 3):
        out, lse = c.attend(0, q, window=window)
        assert torch.isfinite(lse).all()
        want = torch.zeros(Q, H, D, dtype=torch.bool, device=DEV)
        for i in range(Q):
            for t, ch in at.items():
                if t <= i and (window == 0 or t > i - window):
                    want[i, :, ch // 16 * 16:ch // 16 * 16 + 16] = True
        assert torch.equal(out[0].isnan(), want)
