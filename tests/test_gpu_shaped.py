"""Verification under penalties, biases and masks: equal to the definition, computed operation by operation in float32."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from tests.test_gpu_cache_attend import DEV, _i32

pytestmark = pytest.mark.gpu
f32 = np.float32


def _pack(bits):
    """bool [n, V] -> int32 [n, ceil(V / 32)]."""
    n, V = bits.shape
    x = np.zeros((n, -(-V // 32) * 32), bool)
    x[:, :V] = bits
    return np.packbits(x.reshape(n, -1, 32), axis=-1, bitorder="little").view(np.uint32).reshape(n, -1).view(np.int32)


def _choice(x, told, said, rep, pres, freq, bias, ok):
    """Row [V] of float32 -> (choice, its value)."""
    with np.errstate(all="ignore"):
        hit = told | (said > 0)
        x = np.where(hit, np.where(x > 0, x / f32(rep), x * f32(rep)), x)
        x = np.where(said > 0, (x - f32(freq) * said.astype(f32)) - f32(pres), x)
        x = x + bias
    good = ok & (x > -np.inf)
    if good.any():
        best = x[good].max()
        return int(np.flatnonzero(good & (x == best))[0]), best
    return (int(np.flatnonzero(ok)[0]) if ok.any() else -1), f32(-np.inf)


class Case:
    """Random logits with ties, histories, drafts, and whatever of the rest is asked for."""

    def __init__(self, rng, B, K, V, said=20, penalties="usual", n_bias=0, masks=0, offset=0, pad=0, streams=None, special=True, share=0.9):
        self.B, self.K, self.V, self.rng = B, K, V, rng
        n_streams = B if streams is None else max(max(streams) + 1, 1)
        rows = B * (K + 1)
        self.stride = V + pad
        flat = np.full(offset + rows * self.stride, 300.0, f32)            # between the rows lies what would win
        x = np.round(rng.standard_normal((rows, V)) * 4) / 2                # coarse: many ties
        if special and V > 4:
            x[rng.random((rows, V)) < 0.02] = np.nan
            x[rng.random((rows, V)) < 0.02] = -np.inf
            x[rng.random((rows, V)) < 0.02] = -0.0
        for r in range(rows):
            flat[offset + r * self.stride:offset + r * self.stride + V] = x[r]
        self.x = x.astype(f32).reshape(B, K + 1, V)
        self.flat = torch.from_numpy(flat).to(DEV, torch.bfloat16)
        self.logits = self.flat.data_ptr() + 2 * offset
        self.drafts = rng.integers(0, V, size=(B, K)).astype(np.int32)
        self.drafts[rng.random((B, K)) < 0.1] = -1
        if K > 2:
            self.drafts[:, 2] = self.drafts[:, 0]                           # the same token twice
        self.n_draft = rng.integers(0, K + 1, size=B).astype(np.int32)
        self.streams = streams
        self.said = np.zeros((n_streams, V), np.int64)
        self.told = np.zeros((n_streams, V), bool)
        for s in range(n_streams):
            np.add.at(self.said[s], rng.integers(0, V, size=said), 1)
            self.told[s, rng.integers(0, V, size=said)] = True
        self.rep = self.pres = self.freq = None
        if penalties:
            lo, hi = (1.0, 1.5) if penalties == "usual" else (0.5, 2.0)
            self.rep = rng.uniform(lo, hi, B).astype(f32)
            self.pres = rng.uniform(0 if penalties == "usual" else -1, 1, B).astype(f32)
            self.freq = rng.uniform(0 if penalties == "usual" else -0.5, 0.5, B).astype(f32)
        self.bias_t = rng.integers(-2, V + 2, size=(B, n_bias)).astype(np.int32)
        if n_bias > 3:
            self.bias_t[:, 3] = self.bias_t[:, 1]                           # the same token twice
        self.bias_v = (rng.standard_normal((B, n_bias)) * 3).astype(f32)
        self.n_bias = rng.integers(-1, n_bias + 3, size=B).astype(np.int32)
        self.masks = rng.random((masks, V)) < np.where(rng.random((masks, 1)) < 0.5, share, 2.0 / V) if masks else None
        if masks > 1:
            self.masks[1] = False                                           # nothing is allowed
        self.mask_of = rng.integers(-2, masks + 2, size=(B, K + 1)).astype(np.int32)

    def shape(self):
        t = {}
        if self.rep is not None:
            counts = np.where(self.told, self.said - (1 << 31), self.said).astype(np.int32)
            t.update(counts=torch.from_numpy(counts).to(DEV), seen=torch.from_numpy(_pack(counts != 0)).to(DEV))
            t.update({n: torch.from_numpy(v).to(DEV) for n, v in (("repetition", self.rep), ("presence", self.pres), ("frequency", self.freq)) if v is not None})
        if self.bias_t.shape[1]:
            t.update(bias_tokens=_i32(self.bias_t), bias_values=torch.from_numpy(self.bias_v).to(DEV), n_bias=_i32(self.n_bias))
        if self.masks is not None:
            t.update(masks=torch.from_numpy(_pack(self.masks)).to(DEV), mask_of=_i32(self.mask_of))
        return S.SamShape(self.V, **t)

    def want(self):
        B, K, V = self.B, self.K, self.V
        choice, value = np.zeros((B, K + 1), np.int64), np.zeros((B, K + 1), f32)
        for b in range(B):
            s = b if self.streams is None else self.streams[b]
            known = 0 <= s < len(self.said) and self.rep is not None
            said = self.said[s].copy() if known else np.zeros(V, np.int64)
            told = self.told[s] if known else np.zeros(V, bool)
            bias = np.zeros(V, f32)
            for t, v in zip(self.bias_t[b][:max(self.n_bias[b], 0)], self.bias_v[b]):
                if 0 <= t < V:
                    bias[t] += v
            for j in range(K + 1):
                if j and self.rep is not None and 0 <= self.drafts[b, j - 1] < V:
                    said[self.drafts[b, j - 1]] += 1
                m = self.mask_of[b, j]
                ok = self.masks[m] if self.masks is not None and 0 <= m < len(self.masks) else np.ones(V, bool)
                r, p, f = (1.0, 0.0, 0.0) if self.rep is None else (self.rep[b], 0.0 if self.pres is None else self.pres[b], 0.0 if self.freq is None else self.freq[b])
                choice[b, j], value[b, j] = _choice(self.x[b, j], told, said, r, p, f, bias, ok)
        return choice, value

    def run(self, keys=None):
        B, K, V = self.B, self.K, self.V
        keys = torch.full((B * (K + 1),), -1, dtype=torch.int64, device=DEV) if keys is None else keys
        argmax, accepted = (torch.zeros(B, K + 1, dtype=torch.int32, device=DEV) for _ in range(2))
        n_acc, values = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, K + 1, device=DEV)
        drafts, n_draft = _i32(self.drafts), _i32(self.n_draft)
        S.sam_argmax_shaped(self.logits, self.stride, B, K, V, drafts, self.shape(), keys, streams=None if self.streams is None else _i32(self.streams))
        S.sam_verify_from_keys(keys, B, K, drafts, n_draft, argmax, accepted, n_acc, values=values)
        assert not keys.any()
        return argmax.cpu().numpy(), values.cpu().numpy(), accepted.cpu().numpy(), n_acc.cpu().numpy()

    def check(self):
        argmax, values, accepted, n_acc = self.run()
        choice, value = self.want()
        assert (argmax == choice).all()
        assert (values == value).all()                                      # -0 equals 0
        for b in range(self.B):
            a = 0
            while a < self.n_draft[b] and self.drafts[b, a] == choice[b, a]:
                a += 1
            assert n_acc[b] == a + 1
            assert accepted[b].tolist() == self.drafts[b, :a].tolist() + [choice[b, a]] + [-1] * (self.K - a)


@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 31, 32, 33, 100, 8191, 8192, 8193, 20011])
def test_vocabularies(V):
    for kw in (dict(), dict(n_bias=5), dict(masks=4, n_bias=2), dict(penalties=None, masks=3)):
        Case(np.random.default_rng(V), 3, 4, V, said=min(20, V), **kw).check()


@pytest.mark.parametrize("penalties", [None, "usual", "any"])
@pytest.mark.parametrize("n_bias", [0, 1, 300, 512])
@pytest.mark.parametrize("masks", [0, 5])
def test_everything(penalties, n_bias, masks):
    Case(np.random.default_rng(n_bias + masks), 5, 8, 3001, said=200, penalties=penalties, n_bias=n_bias, masks=masks).check()


@pytest.mark.parametrize("offset,pad", [(0, 0), (0, 7), (1, 0), (3, 5), (7, 1)])
@pytest.mark.parametrize("V", [65, 9000])
def test_unaligned_rows(offset, pad, V):
    Case(np.random.default_rng(offset), 3, 3, V, n_bias=4, masks=3, offset=offset, pad=pad).check()


@pytest.mark.parametrize("B,K", [(1, 1), (1, 32), (40, 16), (300, 1)])
def test_batches(B, K):
    Case(np.random.default_rng(B), B, K, 517, n_bias=3, masks=6).check()


def test_streams_named_in_any_order():
    Case(np.random.default_rng(1), 6, 3, 999, said=400, streams=[3, 0, 3, 77, -1, 1]).check()


def test_the_most_said_token_loses():
    """What the model wants most was said: the penalties decide, row by row along the draft."""
    c = Case(np.random.default_rng(2), 4, 4, 5000, said=3000, special=False)
    for b in range(4):
        t = int(np.argmax(c.said[b]))
        c.drafts[b] = t
        c.x[b, :, t] = 9.0
    c.flat.copy_(torch.from_numpy(c.x.reshape(-1)))
    c.check()


def test_rows_of_nothing():
    """Rows of minus infinity, of NaN, masked altogether, and biases of either infinity."""
    c = Case(np.random.default_rng(3), 2, 3, 300, n_bias=4, masks=3, special=False)
    c.x[0, 0], c.x[0, 1], c.x[1, 2] = -np.inf, np.nan, np.inf
    c.x[0, 0, 17] = np.nan
    c.flat.copy_(torch.from_numpy(c.x.reshape(-1)))
    c.mask_of[:] = -1
    c.mask_of[1, 0], c.mask_of[0, 2] = 1, 0
    c.bias_t[1], c.bias_v[1], c.n_bias[1] = [5, 6, 7, 7], [math.inf, -math.inf, math.inf, -math.inf], 4
    c.bias_t[0], c.bias_v[0], c.n_bias[0] = [5, 6, 7, 8], [-math.inf] * 4, 4
    c.check()
    assert c.run()[0][1, 0] == -1


def test_without_anything_it_is_the_plain_argmax():
    rng = np.random.default_rng(4)
    c = Case(rng, 7, 5, 4001, penalties=None, special=False)
    keys = torch.zeros(7 * 6 + 1, dtype=torch.int64, device=DEV)
    S.sam_argmax_partial(c.logits, c.stride, 42, c.V, 0, keys)
    argmax, accepted = (torch.zeros(7, 6, dtype=torch.int32, device=DEV) for _ in range(2))
    n_acc, values = torch.zeros(7, dtype=torch.int32, device=DEV), torch.zeros(7, 6, device=DEV)
    S.sam_verify_from_keys(keys, 7, 5, _i32(c.drafts), _i32(c.n_draft), argmax, accepted, n_acc, values=values)
    got = c.run()
    for x, y in zip((argmax, values, accepted, n_acc), got):
        assert (x.cpu().numpy() == y).all()
    c.check()


def test_a_whole_vocabulary():
    Case(np.random.default_rng(5), 4, 3, 151936, said=5000, n_bias=100, masks=4, special=False).check()


# ------------------------------------------------------------------ histories
def test_history():
    rng = np.random.default_rng(6)
    V, n = 1001, 5
    h = S.SamHistory(n, V, device=DEV)
    said, told = np.zeros((n, V), np.int64), np.zeros((n, V), bool)

    def check():
        counts = np.where(told, said - (1 << 31), said)
        assert (h.counts.cpu().numpy() == counts).all() and (h.seen.cpu().numpy() == _pack(counts != 0)).all()
    for step in range(6):
        B, ld = (n, 40) if step % 2 else (7, 900)
        streams = None if step % 2 else [4, 0, 99, -1, 0, 2, 4]                 # named twice, unknown
        tokens = rng.integers(-3, V + 3, size=(B, ld))
        tokens[:, ::7] = 5
        cnt = rng.integers(-1, ld + 3, size=B)
        h.add(_i32(tokens), n=None if step == 3 else _i32(cnt), streams=None if streams is None else _i32(streams), told=step == 2)
        for b in range(B):
            s = b if streams is None else streams[b]
            if 0 <= s < n:
                for t in tokens[b, :ld if step == 3 else max(min(cnt[b], ld), 0)]:
                    if 0 <= t < V:
                        if step == 2:
                            told[s, t] = True
                        else:
                            said[s, t] += 1
        check()
    h.fork(_i32([0, 2, 50, 1]), _i32([3, 1, 4, -2]))
    for a, z in ((0, 3), (2, 1)):
        said[z], told[z] = said[a], told[a]
    check()
    h.reset(_i32([0, 2, 7]))
    said[[0, 2]], told[[0, 2]] = 0, False
    check()
