"""A small decoder over the paged 4-bit cache, with drafts from agent memory: every cache call as a serving loop uses it.

The model is a stand-in (random weights, a few attention layers, tied embedding); what runs in the library is everything
around its matrix products: the pages of the step (`reserve`), keys and values (`append`), attention over the cache
(`attend`), verification and the next draft (`sam_step_ex`), and what of the step is kept (`commit`).

    python -m harness.cached_decode

decodes a session without memory, indexes what it said, then serves several sessions that fork from one prompt and draft
from that memory; prints how many tokens a step committed.  Then a model with rotated positions does the same over
selected blocks of its context, and under penalties for what was said before.
"""
from __future__ import annotations

import numpy as np
import torch

import paper_2512_18337_b200 as S

DROP = -(1 << 31)


class TinyDecoder:
    """Attention layers with residuals; no positions but the causal mask, or with rope_base queries and keys that are rotated
    to theirs."""

    def __init__(self, vocab=1000, layers=2, heads=8, kv_heads=2, head_dim=128, width=256, seed=0, device="cuda:0",
                 rope_base=None):
        g = torch.Generator().manual_seed(seed)

        def w(*shape):
            return (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to(device, torch.bfloat16)
        self.vocab, self.layers, self.heads, self.kv_heads, self.head_dim = vocab, layers, heads, kv_heads, head_dim
        self.embed = w(vocab, width) * width ** 0.5
        self.qkv = [w((heads + 2 * kv_heads) * head_dim, width) for _ in range(layers)]
        self.out = [w(width, heads * head_dim) for _ in range(layers)]
        self.inv_freq = None if rope_base is None else rope_base ** (-np.arange(0, head_dim, 2) / head_dim)
        self.rope = None if rope_base is None else S.SamRope(self.inv_freq, device=device)

    @staticmethod
    def norm(x):
        return torch.nn.functional.rms_norm(x, x.shape[-1:])

    def forward(self, cache: S.SamCache, tokens, n_new, streams=None, bounds: S.SamBounds | None = None, n_blocks=0):
        """tokens int32 [B, Q]: appends their keys and values to the cache and returns logits bf16 [B, Q, vocab].  With
        bounds, the tokens of a row share n_blocks blocks of the context that they attend to."""
        x = self.embed[tokens.clamp(0, self.vocab - 1).long()]
        B, Q = tokens.shape
        for i in range(self.layers):
            y = (self.norm(x) @ self.qkv[i].T).view(B, Q, -1, self.head_dim)
            q, k, v = y.split([self.heads, self.kv_heads, self.kv_heads], 2)
            if self.rope is None:
                cache.append(i, k, v, n_new=n_new, streams=streams)
            else:
                q = cache.append_rotated(i, q, k, v, self.rope, n_new=n_new, streams=streams)
            if bounds is None:
                o, _ = cache.attend(i, q, n_new=n_new, streams=streams)
            else:
                bounds.update(i, Q, n_new=n_new, streams=streams)
                # a chunk of a prompt is longer than the blocks that a list has to hold of it
                share = min(Q, (n_blocks - 3) * cache.page_tokens + 1)
                blocks = bounds.select(i, q, n_blocks, share=share, n_new=n_new, streams=streams)
                o, _ = cache.attend_blocks(i, q, blocks, share=share, n_new=n_new, streams=streams)
            x = x + o.reshape(B, Q, -1) @ self.out[i].T
        return self.norm(x) @ self.embed.T


class CachedDecoder:
    """Greedy decoding of B streams with drafts of up to K tokens from a SamIndex (or none).

    n_blocks > 0: attention over so many selected blocks of the context (at least 4: one sink, two recent, one more that a
    proposal runs into).  penalties: (repetition, presence, frequency) for what the prompt told and the stream said."""

    def __init__(self, model: TinyDecoder, B: int, K: int, n_pages: int, page_tokens=16, max_pages=64, min_match=2,
                 index: S.SamIndex | None = None, device="cuda:0", n_blocks: int = 0, penalties=None):
        i32 = dict(dtype=torch.int32, device=device)
        self.model, self.B, self.K, self.min_match, self.index = model, B, K, min_match, index
        self.cache = S.SamCache(n_pages, page_tokens, B, max_pages, model.layers, model.kv_heads, model.head_dim, 0, -3,
                                device=device)
        self.state, self.mlen = torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.drafts, self.n_draft = torch.full((B, K), -1, **i32), torch.zeros(B, **i32)
        self.argmax, self.accepted = torch.zeros((B, K + 1), **i32), torch.zeros((B, K + 1), **i32)
        self.n_accepted = torch.zeros(B, **i32)
        self.pending = torch.zeros(B, **i32)       # committed, but not in the cache yet
        self.counters = torch.zeros(S.SAM_N_COUNTERS, dtype=torch.int64, device=device)
        n = S.sam_workspace_bytes(B, K)
        self.ws = torch.zeros(n, dtype=torch.uint8, device=device)
        self.n_blocks = n_blocks
        self.bounds = S.SamBounds(self.cache) if n_blocks else None
        self.history = self.shape = None
        if penalties is not None:
            self.history = S.SamHistory(B, model.vocab, device=device)
            names = ("repetition", "presence", "frequency")
            self.shape = S.SamShape(model.vocab, counts=self.history.counts, seen=self.history.seen, **{
                n: torch.full((B,), float(p), device=device) for n, p in zip(names, penalties)})
            self.keys = torch.zeros(B * (K + 1), dtype=torch.int64, device=device)

    def prompt(self, tokens: np.ndarray, stream: int = 0):
        """The prompt of one stream, but for its last token, into the cache."""
        t = torch.from_numpy(np.ascontiguousarray(tokens[None, :-1], dtype=np.int32)).to(self.pending.device)
        one = torch.tensor([stream], dtype=torch.int32, device=t.device)
        n = torch.tensor([t.shape[1]], dtype=torch.int32, device=t.device)
        self.cache.reserve(n, streams=one)
        self.check()
        self.model.forward(self.cache, t, n, streams=one, bounds=self.bounds, n_blocks=self.n_blocks)
        self.cache.commit(n, streams=one)
        self.pending[stream] = int(tokens[-1])
        if self.history is not None:
            told = torch.from_numpy(np.ascontiguousarray(tokens[None], dtype=np.int32)).to(t.device)
            self.history.add(told, streams=one, told=True)
        if self.index is not None:                 # the automaton has read the prompt too
            self.feed(torch.nn.functional.pad(torch.from_numpy(np.ascontiguousarray(tokens, dtype=np.int32))[None],
                                              (0, 0, stream, self.B - 1 - stream)).to(t.device),
                      torch.nn.functional.pad(n + 1, (stream, self.B - 1 - stream)))

    def check(self):
        """A refused call shows in the cache's status only; what is computed after it does not stand."""
        n_free, status = self.cache.status()
        if status:
            names = [n for n in ("OUT_OF_PAGES", "TABLE_FULL", "BAD_FORK", "GAVE_UP") if status & getattr(S, "SAM_CACHE_" + n)]
            raise RuntimeError(f"the cache refused a call: {', '.join(names)} ({n_free} free pages)")

    def feed(self, tokens, n):
        S.sam_draft(self.index.handle, self.B, self.state, self.mlen, tokens.contiguous(), tokens.shape[1], n, self.K,
                    self.min_match, self.drafts, self.n_draft)

    def fork(self, src: int, dst):
        """Streams dst go on from where src is; they share its pages until one of them writes."""
        d = torch.tensor(dst, dtype=torch.int32, device=self.pending.device)
        self.cache.fork(torch.full_like(d, src), d)
        if self.history is not None:
            self.history.fork(torch.full_like(d, src), d)
        for t in (self.pending, self.state, self.mlen, self.drafts, self.n_draft):
            t[d.long()] = t[src].clone()

    def step(self):
        """One verification step of all streams; returns (tokens [B, K+1], counts [B]) on the device.  They stand if check()
        finds nothing."""
        rows = torch.cat([self.pending[:, None], self.drafts], 1)
        n_new = self.n_draft + 1
        self.cache.reserve(n_new)
        logits = self.model.forward(self.cache, rows, n_new, bounds=self.bounds, n_blocks=self.n_blocks)
        if self.shape is not None:
            S.sam_argmax_shaped(logits, logits.shape[-1], self.B, self.K, self.model.vocab, self.drafts, self.shape,
                                self.keys)
            if self.index is not None:
                S.sam_step_from_keys(self.index.handle, self.keys, self.B, self.K, self.drafts, self.n_draft, self.argmax,
                                     self.accepted, self.n_accepted, self.state, self.mlen, self.min_match, self.drafts,
                                     self.n_draft)
            else:
                S.sam_verify_from_keys(self.keys, self.B, self.K, self.drafts, self.n_draft, self.argmax, self.accepted,
                                       self.n_accepted)
            self.history.add(self.accepted, n=self.n_accepted)
            self.count(n_new - 1)
        elif self.index is not None:
            S.sam_step_ex(self.index.handle, logits, logits.shape[-1], self.B, self.K, self.model.vocab, self.drafts,
                          self.n_draft, self.argmax, self.accepted, self.n_accepted, self.state, self.mlen, self.min_match,
                          self.drafts, self.n_draft, 0, self.counters, self.ws, self.ws.numel())
        else:
            S.sam_verify(logits, logits.shape[-1], self.B, self.K, self.model.vocab, self.drafts, self.n_draft, self.argmax,
                         self.accepted, self.n_accepted, self.ws, self.ws.numel())
        # the rows of the pending token and of the accepted drafts stay; the rest is overwritten by the next step
        self.cache.commit(self.n_accepted)
        last = (self.n_accepted - 1).clamp(min=0).long()[:, None]
        self.pending.copy_(self.accepted.gather(1, last)[:, 0])
        return self.accepted, self.n_accepted

    def count(self, proposed):
        """The counters of sam_step_ex for a step that was verified from keys; proposed: drafts of each stream."""
        committed = self.n_accepted.sum()
        per_call = torch.full_like(committed, self.B)
        self.counters += torch.stack([per_call, committed, proposed.sum(), committed - self.B, (proposed > 0).sum(),
                                      per_call * (self.K + 1)])

    def decode(self, steps: int):
        out = [[] for _ in range(self.B)]
        for _ in range(steps):
            t, n = (x.cpu().numpy() for x in self.step())
            self.check()
            for b in range(self.B):
                out[b] += t[b, :n[b]].tolist()
        return out

    def drop(self, streams):
        s = torch.tensor(streams, dtype=torch.int32, device=self.pending.device)
        self.cache.commit(torch.full_like(s, DROP), streams=s)
        if self.history is not None:
            self.history.reset(s)

    def compact(self):
        self.cache.compact()
        if self.bounds is not None:
            self.bounds.rebuild()              # pages have moved


def main() -> None:
    model = TinyDecoder()
    rng = np.random.default_rng(0)
    prompt = rng.integers(0, model.vocab, size=150)
    first = CachedDecoder(model, B=1, K=1, n_pages=64)
    first.prompt(prompt)
    said = first.decode(200)[0]
    index = S.SamIndex(np.concatenate([prompt, said]).astype(np.int32), [model.vocab])
    B = 4
    d = CachedDecoder(model, B=B, K=8, n_pages=96, index=index)
    d.prompt(prompt)
    d.fork(0, list(range(1, B)))
    free_before, _ = d.cache.status()
    outs = d.decode(30)
    free_after, status = d.cache.status()
    c = d.counters.cpu().numpy()
    print(f"{B} sessions from one prompt: {sum(map(len, outs))} tokens in 30 steps, {c[1] / max(c[0], 1):.2f} per pass; "
          f"free pages {free_before} -> {free_after}, status {status}; as said before: "
          f"{sum(a == b for a, b in zip(outs[0], said))} of {min(len(outs[0]), len(said))}")
    d.drop([1, 3])
    d.cache.compact()
    print(f"after two sessions left and the pool was closed up: {d.cache.status()[0]} free pages")

    model = TinyDecoder(rope_base=10000.0)
    d = CachedDecoder(model, B=B, K=8, n_pages=200, index=index, n_blocks=6, penalties=(1.2, 5.0, 10.0))
    d.prompt(np.concatenate([prompt, said, prompt]))
    d.fork(0, list(range(1, B)))
    outs = d.decode(30)
    print(f"with positions, 6 of up to {-(-int(d.cache.seq_len.max()) // 16)} blocks and penalties: "
          f"{sum(map(len, outs))} tokens in 30 steps, {len(set(outs[0]))} different ones of {len(outs[0])}; "
          f"status {d.cache.status()[1]}")


if __name__ == "__main__":
    main()
