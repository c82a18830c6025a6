"""Weights far below the largest one, in attention over listed blocks: they keep the 11 bits of their type."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from tests.test_gpu_cache_attend import DEV, _i32

pytestmark = pytest.mark.gpu

# A weight is rounded to fp16 and so is the result: 2^-11 each, and 2^-22 for their product.  32-bit sums of 128 numbers of one size,
# the exponential, and a score of up to 22 (as a power of two, off by 2^-23 of itself twice): less than 2^-15 of the result.
BOUND = 2.0 ** -10 + 2.0 ** -15


@pytest.mark.parametrize("Q", [1, 2, 5, 17, 33])
def test_small_weights_keep_their_bits(Q):
    """One position with all of the weight and a value of zero, 127 that have 2^-18.2 to 2^-20.9 of it and a value of 64."""
    H, D, P, T = 8, 128, 16, 128
    c = S.SamCache(32, P, 1, 32, 1, 1, D, 0, -3, device=DEV)
    k, v = torch.zeros(1, 200, 1, D), torch.full((1, 200, 1, D), 64.0)
    k[0, 0, 0, 0] = 6.0
    v[0, 0] = 0.0
    c.reserve(_i32([200 + Q]))
    c.append(0, k.to(DEV, torch.float16), v.to(DEV, torch.float16))
    c.commit(_i32([200]))
    q = torch.zeros(1, Q, H, D, dtype=torch.float16, device=DEV)
    size = torch.linspace(18.2, 20.9, Q * H, dtype=torch.float64) * np.log(2.0) / 6.0
    q[0, :, :, 0] = size.view(Q, H).to(DEV, torch.float16)
    blocks = torch.arange(T // P, dtype=torch.int32, device=DEV).view(1, 1, 1, -1)
    out, lse = c.attend_blocks(0, q, blocks, share=Q, scale=1.0)
    w = torch.exp(-6.0 * q[0, :, :, 0].double())[..., None]
    held = c.read(0, first=_i32([0]), n=_i32([T]), max_n=T, dtype=torch.float16)      # 64 has no code of its own: its nearest is held
    value = float(held[1][0, 1, 0, 0])
    assert (held[1][0, 1:] == value).all() and not held[1][0, 0].any() and held[0].double().sum() == 6
    want = (T - 1) * value * w / (1 + (T - 1) * w)
    assert ((out[0].double() - want).abs() <= BOUND * want).all()
    assert (lse[0].double() - (6.0 * q[0, :, :, 0].double() + torch.log1p((T - 1) * w[..., 0]))).abs().max() < 2.0 ** -18
    assert c.status()[1] == 0
