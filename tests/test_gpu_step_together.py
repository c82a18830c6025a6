"""Rotated appends, selected blocks and shaped verification as a decoding step has them: against a model without the cache in
64 bits, recorded in a graph, on streams of their own, and with pages that move."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from harness.cached_decode import CachedDecoder, TinyDecoder
from tests import cache_reference as R
from tests.test_gpu_cache_attend import DEV, _i32

pytestmark = pytest.mark.gpu


def _rotate(x, pos, f):
    """x [T, H, D] in 64 bits."""
    a = np.asarray(pos, np.float64)[:, None] * f
    cos, sin, h = np.cos(a)[:, None], np.sin(a)[:, None], x.shape[-1] // 2
    return np.concatenate([x[..., :h] * cos - x[..., h:] * sin, x[..., h:] * cos + x[..., :h] * sin], -1)


def _logits(model: TinyDecoder, tokens):
    """64-bit logits [T, vocab] of a token sequence, with full attention over keys and values in four bits."""
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
        q, k = (_rotate(t, range(T), model.inv_freq) for t in (q, k))
        k, v = (R.values(*R.quantise(t, e), e) for t, e in ((k, 0), (v, -3)))
        o = R.attend(q, k, v, np.ones(T, bool), 0, T, H // Hkv, D ** -0.5, 0)[0]
        x = x + o.reshape(T, -1) @ f(model.out[i]).T
    return norm(x) @ f(model.embed).T


PENALTIES = (1.3, 0.2, 0.1)


def _shape(logits, told, said):
    """Rows of logits under the penalties; said grows token by token."""
    out = logits.copy()
    counts = np.zeros(logits.shape[1])
    for i in range(len(logits)):
        hit = told | (counts > 0)
        out[i][hit] = np.where(out[i][hit] > 0, out[i][hit] / PENALTIES[0], out[i][hit] * PENALTIES[0])
        out[i] -= PENALTIES[2] * counts + PENALTIES[1] * (counts > 0)
        if i < len(said):
            counts[said[i]] += 1
    return out


@pytest.mark.parametrize("n_blocks", [0, 64])
@pytest.mark.parametrize("penalties", [None, PENALTIES])
def test_decoding_follows_the_model(n_blocks, penalties):
    """With as many blocks as there are the selection leaves nothing out: both attentions follow the same model."""
    model = TinyDecoder(vocab=300, width=128, rope_base=10000.0)
    rng = np.random.default_rng(0)
    prompt = rng.integers(0, model.vocab, size=60)
    first = CachedDecoder(model, B=1, K=1, n_pages=32, n_blocks=n_blocks, penalties=penalties)
    first.prompt(prompt)
    said = first.decode(50)[0]
    index = S.SamIndex(np.concatenate([prompt, said]).astype(np.int32), [model.vocab])
    d = CachedDecoder(model, B=3, K=8, n_pages=60, index=index, n_blocks=n_blocks, penalties=penalties)
    d.prompt(prompt)
    d.fork(0, [1, 2])
    outs = d.decode(12)
    assert d.cache.status()[1] == 0
    assert outs[1] == outs[0] and outs[2] == outs[0]
    assert len(outs[0]) > 18                                     # drafts from memory are accepted
    told = np.zeros(model.vocab, bool)
    told[prompt] = True
    for tokens in (said, outs[0]):
        ids = np.concatenate([prompt, tokens]).astype(np.int64)
        ref = _logits(model, ids[:-1])[len(prompt) - 1:]
        size = np.abs(ref).max(-1)
        if penalties:
            ref = _shape(ref, told, tokens)
        # the loop computes in bf16 between the layers: its choice may trail the best by that much of the logits' size
        best, chosen = ref.max(-1), ref[np.arange(len(tokens)), tokens]
        assert (best - chosen <= 0.1 * size).all()
        assert (ref.argmax(-1) == tokens).mean() > 0.8
    if penalties:
        counts = d.history.counts.cpu().numpy()
        want = np.bincount(outs[0], minlength=model.vocab) + np.where(told, -(1 << 31), 0)
        assert (counts == want).all()


def test_few_blocks_and_pages_that_move():
    """Sessions over selected blocks go on the same after other sessions left and the pool was closed up."""
    model = TinyDecoder(vocab=300, width=128, rope_base=10000.0)
    prompt = np.random.default_rng(1).integers(0, model.vocab, size=400)

    def go(close):
        d = CachedDecoder(model, B=3, K=1, n_pages=160, n_blocks=8)
        for s in (1, 0, 2):
            d.prompt(prompt[s:], stream=s)
        a = d.decode(10)
        d.drop([1])
        if close:
            d.compact()
            assert int(d.cache.page_table[[0, 2]].max()) < int((d.cache.ref_count > 0).sum())
        b = d.decode(20)
        assert d.cache.status()[1] == 0
        return [x + y for x, y in zip(a, b)]
    kept, moved = go(False), go(True)
    assert kept[0] == moved[0] and kept[2] == moved[2]


class Step:
    """One layer's calls and the verification of a step, over tensors that stay."""

    def __init__(self, seed, lengths, Q=5, H=8, Hkv=2, D=128, P=16, V=3000, n_blocks=8, stream=None):
        rng = np.random.default_rng(seed)
        B = self.B = len(lengths)
        self.Q, self.V, self.stream, self.n_blocks = Q, V, stream, n_blocks
        held = [-(-(l + Q) // P) for l in lengths]
        self.cache = S.SamCache(sum(held), P, B, max(held), 1, Hkv, D, 0, -3, device=DEV, stream=stream)
        self.bounds = S.SamBounds(self.cache, stream=stream)
        self.rope = S.SamRope(10000.0 ** (-np.arange(D // 2) * 2 / D), device=DEV, stream=stream)
        with S.SamCache._on(DEV, stream):
            self.cache.pages.copy_(torch.from_numpy(rng.integers(0, 256, size=self.cache.pages.shape, dtype=np.uint8)))
            self.cache.pages[..., 16 * D:].clamp_(max=0x37)
            table, at = -np.ones((B, max(held)), np.int32), 0
            for s, n in enumerate(held):
                table[s, :n] = np.arange(at, at + n)
                at += n
            self.cache.page_table.copy_(torch.from_numpy(table))
            self.cache.seq_len.copy_(_i32(lengths))
            self.qkv = torch.from_numpy(rng.standard_normal((B, Q, H + 2 * Hkv, D))).to(DEV, torch.bfloat16)
            self.q, self.k, self.v = self.qkv.split([H, Hkv, Hkv], 2)
            self.n_new = _i32(rng.integers(1, Q + 1, size=B))
            self.logits = torch.from_numpy(rng.standard_normal((B * Q, V))).to(DEV, torch.bfloat16)
            self.drafts, self.n_draft = _i32(rng.integers(0, V, size=(B, Q - 1))), self.n_new - 1
            self.history = S.SamHistory(B, V, device=DEV)
            self.history.add(_i32(rng.integers(0, V, size=(B, 500))))
            ones = torch.ones(B, device=DEV)
            self.shape = S.SamShape(V, counts=self.history.counts, seen=self.history.seen, repetition=1.2 * ones,
                                    presence=0.1 * ones, frequency=0.3 * ones)
            self.keys = torch.zeros(B * Q, dtype=torch.int64, device=DEV)
            self.argmax, self.accepted = (torch.zeros(B, Q, dtype=torch.int32, device=DEV) for _ in range(2))
            self.n_acc, self.values = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, Q, device=DEV)
            self.turned, self.out = torch.empty_like(self.q, memory_format=torch.contiguous_format), torch.empty(B, Q, H, D, dtype=self.q.dtype, device=DEV)
            self.lse = torch.empty(B, Q, H, device=DEV)
            self.blocks = torch.empty(B, 1, Hkv, n_blocks, dtype=torch.int32, device=DEV)
            n = S.sam_cache_select_workspace_bytes(self.cache.handle, B, Q, Q)
            self.ws = torch.empty(n, dtype=torch.uint8, device=DEV)
        self.bounds.rebuild(stream=stream)

    def run(self):
        st, B, K = self.stream, self.B, self.Q - 1
        self.cache.append_rotated(0, self.q, self.k, self.v, self.rope, n_new=self.n_new, out=self.turned, stream=st)
        self.bounds.update(0, self.Q, n_new=self.n_new, stream=st)
        self.bounds.select(0, self.turned, self.n_blocks, share=self.Q, n_new=self.n_new, out=self.blocks, workspace=self.ws, stream=st)
        self.cache.attend_blocks(0, self.turned, self.blocks, share=self.Q, n_new=self.n_new, out=self.out, lse=self.lse, stream=st)
        S.sam_argmax_shaped(self.logits, self.V, B, K, self.V, self.drafts, self.shape, self.keys, stream=st)
        S.sam_verify_from_keys(self.keys, B, K, self.drafts, self.n_draft, self.argmax, self.accepted, self.n_acc, values=self.values, stream=st)
        return [self.turned, self.blocks, self.out, self.lse, self.argmax, self.accepted, self.n_acc, self.values, self.cache.pages, self.bounds.codes]


LENGTHS = [300, 17, 0, 1500, 64]


@pytest.mark.parametrize("Q", [2, 9])
def test_recorded_steps(Q):
    """Replays give what the calls give, also when the first call is a recorded one, and after other calls in between."""
    eager = Step(3, LENGTHS, Q=Q)
    want = [x.clone() for x in eager.run()]
    s = Step(3, LENGTHS, Q=Q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = s.run()
    other = Step(4, [2000] * 20, Q=17, H=16)
    for _ in range(3):
        other.run()
        for x in got[:8]:
            x.fill_(9)
        g.replay()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert s.cache.status()[1] == 0


@pytest.mark.parametrize("how", ["object", "handle"])
def test_steps_on_streams_of_their_own(how):
    """Two steps at once, each on its stream with its tensors."""
    wants = [[x.clone() for x in Step(k, LENGTHS, Q=q).run()] for k, q in ((5, 9), (6, 17))]
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    steps = [Step(k, LENGTHS, Q=q, stream=s if how == "object" else s.cuda_stream) for (k, q), s in zip(((5, 9), (6, 17)), sides)]
    torch.cuda.synchronize()
    gots = []
    for _ in range(10):
        gots = [s.run() for s in steps]
    for s in sides:
        s.synchronize()
    for got, want in zip(gots, wants):
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert all(s.cache.status()[1] == 0 for s in steps)


def test_the_same_call_gives_the_same_bits():
    s = Step(7, [3000, 2900, 5, 700], Q=17, H=16)
    want = [x.clone() for x in s.run()]
    for _ in range(5):
        assert all(torch.equal(x, y) for x, y in zip(s.run(), want))
