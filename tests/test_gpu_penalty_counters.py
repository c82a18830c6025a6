"""The counters of accepted drafts, kept under penalties too."""
from __future__ import annotations

import numpy as np
import pytest

import paper_2512_18337_b200 as S
from harness.cached_decode import CachedDecoder, TinyDecoder

pytestmark = pytest.mark.gpu


def _decode(penalties, index, model, prompt):
    d = CachedDecoder(model, B=3, K=8, n_pages=60, index=index, penalties=penalties)
    d.prompt(prompt)
    d.fork(0, [1, 2])
    return d, d.decode(12)


def test_counters_under_penalties():
    """Penalties that change nothing: the counters are those of the step without.  Others: they fit what was committed, and
    say whether speculation pays."""
    model = TinyDecoder(vocab=300, width=128)
    prompt = np.random.default_rng(0).integers(0, model.vocab, size=60)
    first = CachedDecoder(model, B=1, K=1, n_pages=32)
    first.prompt(prompt)
    index = S.SamIndex(np.concatenate([prompt, first.decode(50)[0]]).astype(np.int32), [model.vocab])
    plain, said = _decode(None, index, model, prompt)
    same, out = _decode((1.0, 0.0, 0.0), index, model, prompt)
    assert out == said and plain.counters.tolist() == same.counters.tolist()
    assert plain.counters[0] == 36 and plain.counters[3] > 0
    d, out = _decode((1.3, 0.2, 0.1), index, model, prompt)
    passes, committed, proposed, accepted, runs, rows = d.counters.tolist()
    assert passes == 36 and committed == sum(map(len, out)) == passes + accepted and rows == passes * 9
    assert accepted <= proposed <= 8 * runs and runs <= passes
    assert S.sam_speculation_pays(d.counters.cpu().numpy(), 8, 0.5)
