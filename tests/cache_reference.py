"""The paged 4-bit cache, plainly and in 64 bits: the format by search over its values, the books as lists that one row
after the other changes, attention as the formula says.  Shares nothing with the library."""
from __future__ import annotations

import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([(m / 8) * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])


def nearest(table, x):
    """Index of the nearest entry of an ascending table, ties to the even index, saturating."""
    hi = np.clip(np.searchsorted(table, x), 1, len(table) - 1)
    lo = hi - 1
    dl, dh = x - table[lo], table[hi] - x
    return np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)


def quantise(x, exp):
    """float64 [..., D] -> (codes [..., D] with the sign as bit 3, scale bytes [..., D/16])."""
    b = np.asarray(x, np.float64).reshape(*x.shape[:-1], -1, 16)
    nan = np.isnan(b).any(-1)
    amax = np.abs(np.where(nan[..., None], 0, b)).max(-1)
    s8 = nearest(E4M3, np.minimum(amax / (6 * 2.0 ** exp), 448.0))
    s = E4M3[s8] * 2.0 ** exp
    with np.errstate(divide="ignore", invalid="ignore"):
        y = np.abs(b) / s[..., None]
    codes = nearest(E2M1, np.minimum(np.nan_to_num(y, nan=0.0, posinf=6.0), 6.0)) + 8 * np.signbit(b)
    codes = np.where(((s > 0) & ~nan)[..., None], codes, 0)
    return codes.reshape(x.shape).astype(np.uint8), np.where(nan, 0x7F, s8).astype(np.uint8)


def values(codes, scales, exp):
    table = np.append(E4M3, np.nan)
    v = np.where(codes & 8, -1.0, 1.0) * E2M1[codes & 7]
    return v * np.repeat(table[scales & 0x7F], 16, -1) * 2.0 ** exp


def unpack_pages(raw, D):
    """uint8 [pages, layers, heads, tiles, 18 D] -> codes [2, pages, layers, heads, tokens, D], scales [2, ..., D/16]."""
    codes, scales = [], []
    for v in range(2):
        c = raw[..., v * 8 * D:(v + 1) * 8 * D].reshape(*raw.shape[:-1], 16, D // 2)
        c = np.stack([c & 15, c >> 4], -1).reshape(*raw.shape[:-1], 16, D)
        s = raw[..., (16 + v) * D:(17 + v) * D].reshape(*raw.shape[:-1], 16, D // 16)
        codes.append(c.reshape(*raw.shape[:3], -1, D))
        scales.append(s.reshape(*raw.shape[:3], -1, D // 16))
    return np.stack(codes), np.stack(scales)


class Books:
    """Tables, counts, free list and page contents (a page is any numpy row)."""

    def __init__(self, n_pages, P, n_streams, max_pages, pages=None):
        self.P, self.max_pages = P, max_pages
        self.table = -np.ones((n_streams, max_pages), np.int32)
        self.len = np.zeros(n_streams, np.int64)
        self.ref = np.zeros(n_pages, np.int32)
        self.free = list(range(n_pages - 1, -1, -1))
        self.status = 0
        self.pages = pages

    def held(self, s):
        return -(-int(self.len[s]) // self.P)

    def reserve(self, rows):
        """rows: [(stream, tokens)] in order."""
        rows = [(s, n) for s, n in rows if n > 0 and 0 <= s < len(self.len)]
        writers = {}
        for s, n in rows:
            i = int(self.len[s]) // self.P
            if self.len[s] % self.P and i < self.max_pages and self.table[s, i] >= 0:
                writers.setdefault(int(self.table[s, i]), []).append(s)
        plan, full = [], False
        for s, n in rows:
            first, want = int(self.len[s]) // self.P, -(-(int(self.len[s]) + n) // self.P)
            full |= want > self.max_pages
            for i in range(first, min(want, self.max_pages)):
                p = int(self.table[s, i])
                if p < 0:
                    plan.append((s, i, None))
                elif i == first and s in writers.get(p, ()) and not (len(writers[p]) == self.ref[p] and writers[p][-1] == s):
                    plan.append((s, i, p))
        if full or len(plan) > len(self.free):
            self.status |= 2 if full else 1
            return
        for s, i, old in plan:
            p = self.free.pop()
            self.table[s, i] = p
            self.ref[p] = 1
            if old is not None:
                self.ref[old] -= 1
                if self.pages is not None:
                    self.pages[p] = self.pages[old]

    def commit(self, rows):
        gone = []
        for s, n in rows:
            if not 0 <= s < len(self.len):
                continue
            self.len[s] = min(max(int(self.len[s]) + n, 0), self.max_pages * self.P)
            i = self.held(s)
            while i < self.max_pages and self.table[s, i] >= 0:
                gone.append(int(self.table[s, i]))
                self.table[s, i] = -1
                i += 1
        for p in gone:
            self.ref[p] -= 1
        for p in dict.fromkeys(gone):
            if self.ref[p] == 0:
                self.free.append(p)

    def fork(self, pairs):
        for a, z in pairs:
            n = len(self.len)
            if not (0 <= a < n and 0 <= z < n) or a == z or self.len[z] or self.table[z, 0] != -1:
                self.status |= 4
                continue
            for i in range(self.held(a)):
                self.table[z, i] = self.table[a, i]
                if self.table[a, i] >= 0:
                    self.ref[self.table[a, i]] += 1
            self.len[z] = self.len[a]

    def compact(self):
        live = [p for p in range(len(self.ref)) if self.ref[p] > 0]
        src = [p for p in live if p >= len(live)]
        dst = [p for p in range(len(live)) if self.ref[p] == 0]
        for a, z in zip(src, dst):
            self.ref[z], self.ref[a] = self.ref[a], 0
            self.table[self.table == a] = z
            if self.pages is not None:
                self.pages[z] = self.pages[a]
        self.free = list(range(len(self.ref) - 1, len(live) - 1, -1))


def attend(q, k, v, present, length, n, g, scale, window):
    """q [Q, H, D], k, v [T, Hkv, D], present [T] in 64 bits -> out, lse, and per row: the mean of |v| under the weights and
    the largest sum of |q k| (what the bounds of the tests are made of)."""
    Q, H, D = q.shape
    out, lse = np.zeros((Q, H, D)), np.full((Q, H), -np.inf)
    mean_abs, size = np.zeros((Q, H, D)), np.zeros((Q, H))
    for i in range(min(n, Q)):
        p = length + i
        lo = max(0, p - window + 1) if window else 0
        on = [j for j in range(lo, min(p + 1, len(present))) if present[j]]
        if not on:
            continue
        for h in range(H):
            kk, vv = k[on, h // g], v[on, h // g]
            s = scale * (kk @ q[i, h])
            w = np.exp(s - s.max())
            out[i, h] = w @ vv / w.sum()
            lse[i, h] = s.max() + math.log(w.sum())
            mean_abs[i, h] = w @ np.abs(vv) / w.sum()
            size[i, h] = abs(scale) * (np.abs(kk) @ np.abs(q[i, h])).max()
    return out, lse, mean_abs, size
