"""Attention recorded in a CUDA graph, next to calls that are not."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from tests.test_gpu_cache_attend import DEV, _cache

pytestmark = pytest.mark.gpu


def _queries(rng, Q):
    return torch.from_numpy(rng.standard_normal((2, Q, 8, 128))).to(DEV, torch.bfloat16)


def _record(c, q, out, lse):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attend(0, q, out=out, lse=lse)
    return g


@pytest.mark.parametrize("first,then", [(1, 64), (64, 1)])
def test_recorded_calls_outlive_larger_ones(first, then):
    """A graph of one size, then a call of the other size, then fresh memory: the replay computes the same and touches nothing else."""
    rng = np.random.default_rng(first)
    c, _, _ = _cache(rng, [3000, 900], [64, 64], 16, 2, 128)
    q, q2 = _queries(rng, first), _queries(rng, then)
    want = [x.clone() for x in c.attend(0, q)]
    want2 = [x.clone() for x in c.attend(0, q2)]
    out, lse = (torch.empty_like(x) for x in want)
    g = _record(c, q, out, lse)
    c.attend(0, q2)
    fresh = [torch.full((n << 20,), 7, dtype=torch.uint8, device=DEV) for n in (4, 8, 9, 16, 21, 32)]
    for _ in range(3):
        out.fill_(9)
        lse.fill_(9)
        g.replay()
        again = c.attend(0, q2)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert torch.equal(again[0], want2[0]) and torch.equal(again[1], want2[1])
    assert all(bool((t == 7).all()) for t in fresh)
    assert c.status()[1] == 0


@pytest.mark.parametrize("Q", [1, 64])
def test_the_first_call_may_be_a_recorded_one(Q):
    """Another call before the first replay finds a workspace that is ready."""
    rng = np.random.default_rng(2)
    c, _, _ = _cache(rng, [3000, 900], [64, 64], 16, 2, 128)
    q = _queries(rng, Q)
    out, lse = torch.empty_like(q), torch.empty(2, Q, 8, device=DEV)
    g = _record(c, q, out, lse)
    eager = c.attend(0, q)
    g.replay()
    assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
    other, _, _ = _cache(np.random.default_rng(2), [3000, 900], [64, 64], 16, 2, 128)
    want = other.attend(0, q)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
