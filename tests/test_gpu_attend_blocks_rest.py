"""Attention over listed blocks with a few query rows behind a full tile of 128: many lists, where another kernel takes them, and few."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from tests.test_gpu_attend_blocks import _compare, _lists
from tests.test_gpu_cache_attend import DEV, DT, _cache, _i32

pytestmark = pytest.mark.gpu

CASES = [
    # streams, Q, H, Hkv, D, share, n_blocks
    (40, 17, 16, 2, 128, 17, 6),       # 136 rows, 80 lists and heads
    (34, 17, 16, 2, 128, 17, 6),       # 68
    (40, 65, 4, 2, 64, 65, 9),         # 130
    (80, 129, 1, 1, 128, 129, 11),     # 129
    (40, 33, 8, 1, 64, 33, 7),         # 264, 40
    (80, 33, 8, 1, 64, 33, 7),         # 264, 80
    (20, 66, 8, 2, 128, 33, 5),        # 132, two lists a row
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_rows_behind_a_full_tile(case, dtype):
    """Streams with all of their tokens, with one less, with fewer than a tile, with none."""
    B, Q, H, Hkv, D, share, n_blocks = CASES[case]
    rng = np.random.default_rng(case)
    lengths = [int(x) for x in rng.integers(0, 300, size=B)]
    n_new = [Q if b % 4 < 2 else Q - 1 if b % 4 == 2 else int(rng.integers(-1, Q)) for b in range(B)]
    c, raw, table = _cache(rng, lengths, [max(n, 0) for n in n_new], 16, Hkv, D, holes=0.05)
    q = torch.from_numpy(rng.standard_normal((B, Q, H, D))).to(DEV, DT[dtype])
    blocks = _lists(rng, lengths, n_new, Q, Hkv, 16, share, n_blocks, table.shape[1])
    out, lse = c.attend_blocks(1, q, _i32(blocks), share=share, n_new=_i32(n_new))
    _compare(c, raw, table, q, blocks, out, lse, lengths, n_new, 16, share, D ** -0.5, dtype, 1)
    for _ in range(3):
        again, lse2 = c.attend_blocks(1, q, _i32(blocks), share=share, n_new=_i32(n_new))
        assert torch.equal(again, out) and torch.equal(lse2, lse)
    assert c.status()[1] == 0
