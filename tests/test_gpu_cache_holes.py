"""Attention over contexts whose pages are partly gone (evicted by the caller), where what is left scores far below zero: an
absent position has no score, so it must not set what the weights are taken relative to."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests.test_gpu_cache_attend import DEV, DT, _cache, _check, _tokens

pytestmark = pytest.mark.gpu


def _scores_around(level, rng, lengths, Q, H, Hkv, D, P, dtype, holes):
    """A cache with keys of 1 and 1.5 and queries below zero: scores of about `level` without a scale, none near zero.
    holes(stream) -> which table entries are gone."""
    c, raw, table = _cache(rng, lengths, [Q] * len(lengths), P, Hkv, D, n_layers=1, garbage=False)
    raw[..., :8 * D] = rng.choice(np.array([0x22, 0x23, 0x32, 0x33], np.uint8), size=raw[..., :8 * D].shape)
    raw[..., 16 * D:17 * D] = 0x38                        # a scale of one
    for s in range(len(lengths)):
        table[s, holes(s)] = -1
    c.pages.copy_(torch.from_numpy(raw))
    c.page_table.copy_(torch.from_numpy(table))
    q = level / (1.25 * D) * rng.uniform(0.9, 1.1, (len(lengths), Q, H, D))
    return c, raw, table, torch.from_numpy(q).to(DEV, DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("level", [-40, -200, 60])
@pytest.mark.parametrize("Q,H,Hkv,D,P", [(40, 2, 2, 128, 16), (17, 8, 2, 64, 64), (150, 1, 1, 128, 32), (9, 8, 2, 128, 16), (1, 4, 2, 64, 16)])
def test_absent_pages_have_no_score(Q, H, Hkv, D, P, level, dtype):
    """Leading pages gone (more than a step of 128 tokens), single pages gone in the middle, all but the last gone."""
    rng = np.random.default_rng(abs(level) + Q)
    lengths = [700, 515, 400]

    def holes(s):
        return [slice(0, -(-192 // P)), slice(1, None, 3), slice(0, (lengths[s] - 1) // P)][s]
    c, raw, table, q = _scores_around(level, rng, lengths, Q, H, Hkv, D, P, dtype, holes)
    out, lse = c.attend(0, q, scale=1.0)
    for b in range(len(lengths)):
        k, v, there = _tokens(raw, table, b, 0, P, D, (0, -3))
        assert not there.all()
        ref = R.attend(q[b].double().cpu().numpy(), k, v, there, lengths[b], Q, H // Hkv, 1.0, 0)
        assert (np.abs(ref[1]) > abs(level) / 2).all()
        _check(out[b], lse[b], ref, dtype, D)
