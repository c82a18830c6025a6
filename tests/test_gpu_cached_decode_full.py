"""The decoding loop does not go on over a cache that has no room."""
from __future__ import annotations

import numpy as np
import pytest

from harness.cached_decode import CachedDecoder, TinyDecoder

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages,max_pages,name", [(4, 64, "OUT_OF_PAGES"), (64, 4, "TABLE_FULL")])
def test_decoding_stops_where_the_pages_end(n_pages, max_pages, name):
    model = TinyDecoder(vocab=300, width=128)
    prompt = np.arange(50) % model.vocab
    d = CachedDecoder(model, B=1, K=1, n_pages=n_pages, max_pages=max_pages)
    d.prompt(prompt)
    assert len(d.decode(10)[0]) == 10                      # 49 + 10 of 64 positions
    with pytest.raises(RuntimeError, match=name):
        d.decode(20)
    room = CachedDecoder(model, B=1, K=1, n_pages=64, max_pages=64)
    room.prompt(prompt)
    assert len(room.decode(30)[0]) == 30


def test_a_prompt_without_room_is_refused():
    d = CachedDecoder(TinyDecoder(vocab=300, width=128), B=2, K=1, n_pages=3)
    with pytest.raises(RuntimeError, match="OUT_OF_PAGES"):
        d.prompt(np.arange(50))


def test_a_refused_fork_is_seen():
    d = CachedDecoder(TinyDecoder(vocab=300, width=128), B=2, K=1, n_pages=30)
    d.prompt(np.arange(50))
    d.fork(0, [1])
    d.fork(0, [1])
    with pytest.raises(RuntimeError, match="BAD_FORK"):
        d.decode(1)
