"""The decoding loop over the 4-bit cache: every committed token is the greedy choice of a model that is computed without
the cache, in 64 bits, over keys and values rounded as the definition says."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from harness.cached_decode import CachedDecoder, TinyDecoder
from tests import cache_reference as R

pytestmark = pytest.mark.gpu


def _logits(model: TinyDecoder, tokens):
    """64-bit logits [T, vocab] of a token sequence."""
    def f(t):
        return t.double().cpu().numpy()

    def norm(x):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + torch.finfo(torch.bfloat16).eps)
    H, Hkv, D = model.heads, model.kv_heads, model.head_dim
    x = f(model.embed)[tokens]
    T = len(tokens)
    for i in range(model.layers):
        y = (norm(x) @ f(model.qkv[i]).T).reshape(T, -1, D)
        q, k, v = y[:, :H], y[:, H:H + Hkv], y[:, H + Hkv:]
        k, v = (R.values(*R.quantise(t, e), e) for t, e in ((k, 0), (v, -3)))
        o = R.attend(q, k, v, np.ones(T, bool), 0, T, H // Hkv, D ** -0.5, 0)[0]
        x = x + o.reshape(T, -1) @ f(model.out[i]).T
    return norm(x) @ f(model.embed).T


def test_decoding_with_memory_follows_the_model():
    model = TinyDecoder(vocab=300, width=128)
    rng = np.random.default_rng(0)
    prompt = rng.integers(0, model.vocab, size=37)
    first = CachedDecoder(model, B=1, K=1, n_pages=32)
    first.prompt(prompt)
    said = first.decode(60)[0]
    index = S.SamIndex(np.concatenate([prompt, said]).astype(np.int32), [model.vocab])
    d = CachedDecoder(model, B=3, K=8, n_pages=40, index=index)
    d.prompt(prompt)
    d.fork(0, [1, 2])
    assert int(d.cache.ref_count.max()) == 3
    outs = d.decode(12)
    n_free, status = d.cache.status()
    assert status == 0
    c = d.counters.cpu().numpy()
    assert c[1] > 1.5 * c[0]                                   # drafts from memory are accepted
    for tokens in (said, outs[0]):
        ids = np.concatenate([prompt, tokens]).astype(np.int64)
        ref = _logits(model, ids[:-1])[len(prompt) - 1:]
        # the loop computes in bf16 between the layers: its choice may trail the best by that much of the logits' size
        best, chosen = ref.max(-1), ref[np.arange(len(tokens)), tokens]
        assert (best - chosen <= 0.1 * np.abs(ref).max(-1)).all()
        assert (ref.argmax(-1) == tokens).mean() > 0.8
    assert outs[1] == outs[0] and outs[2] == outs[0]           # the forks say the same
    # lengths are what was committed; what two streams leave and nobody holds is free again, and the pool closes up
    held = (len(prompt) - 1 + len(outs[0]))
    assert d.cache.seq_len.tolist() == [held] * 3
    d.drop([1, 2])
    live = int((d.cache.ref_count > 0).sum())
    assert live == -(-held // 16)
    d.cache.compact()
    assert d.cache.page_table.max() == live - 1
    more = d.decode(3)                                          # the streams that left start over on page after page of their own
    assert d.cache.status()[1] == 0 and len(more[0]) >= 3
