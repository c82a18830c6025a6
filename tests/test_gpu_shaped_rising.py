"""Shaped verification where all warps of a block raise the best of a row at the same time: the choice is the definition's."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from tests.test_gpu_cache_attend import DEV
from tests.test_gpu_shaped import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("penalties", [None, "usual", "any"])
@pytest.mark.parametrize("masks", [0, 5])
@pytest.mark.parametrize("down", [False, True])
def test_rows_that_rise_everywhere(penalties, masks, down):
    """Every warp finds more than was known when it asked, in rows that rise or fall over the vocabulary, with ties of 64 tokens;
    the same call gives the same words each time."""
    rng = np.random.default_rng(masks)
    c = Case(rng, 6, 7, 40007, said=300, penalties=penalties, n_bias=9, masks=masks, pad=1, special=False)
    rise = np.arange(c.V) // 64 * 0.25
    x = (rise[::-1] if down else rise) - 60.0
    x = torch.from_numpy(np.broadcast_to(x, c.x.shape).astype(np.float32).copy()).to(torch.bfloat16)
    c.x = x.float().numpy()
    c.flat.as_strided((c.B * (c.K + 1), c.V), (c.stride, 1)).copy_(x.view(-1, c.V).to(DEV))
    c.check()
    first = c.run()
    for _ in range(20):
        assert all((a == b).all() for a, b in zip(c.run(), first))
