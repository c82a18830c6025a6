"""A cache that is made and used on a stream of its own, given as an object or as a handle."""
from __future__ import annotations

import pytest
import torch

import paper_2512_18337_b200 as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("how", ["object", "handle", "default"])
def test_a_cache_on_a_stream_of_its_own(how):
    side = torch.cuda.Stream() if how != "default" else torch.cuda.default_stream()
    stream = side if how == "object" else side.cuda_stream
    torch.manual_seed(0)
    k, v = (torch.randn(2, 40, 2, 64, device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.randn(2, 40, 4, 64, device=DEV).to(torch.bfloat16)
    n = torch.full((2,), 40, dtype=torch.int32, device=DEV)

    def go(stream):
        c = S.SamCache(12, 16, 2, 4, 1, 2, 64, device=DEV, stream=stream)
        c.reserve(n, stream=stream)
        c.append(0, k, v, stream=stream)
        out = c.attend(0, q, stream=stream)
        kv = c.read(0, max_n=40, stream=stream)
        c.commit(n, stream=stream)
        status = c.status(stream=stream)
        return c, [*out, *kv, c.seq_len], status
    torch.cuda.synchronize()
    _, want, status = go(None)
    torch.cuda.synchronize()
    c, got, status2 = go(stream)
    assert status == status2 == (6, 0)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
