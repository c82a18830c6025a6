"""Selections and listed attention whose kernels are placed while the one before them ends: recorded behind nothing, behind another
stream and behind a fill, and one call straight after the other with inputs and scratch that change in between."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2512_18337_b200 as S
from tests.test_gpu_attend_blocks import _lists
from tests.test_gpu_cache_attend import DEV, _cache, _i32

pytestmark = pytest.mark.gpu

SHAPES = [  # lengths, Q, H, share: the scores by mma and by tcgen05; attention by one kernel, by the other, and by both
    ([900, 3000, 17, 2047], 1, 8, 1),
    ([900, 3000, 17, 2047], 17, 16, 17),
    ([700, 2500], 65, 8, 16),
]


class Calls:
    def __init__(self, lengths, Q, H, share, seed=0):
        rng = np.random.default_rng(seed)
        self.Q, self.share, self.lengths = Q, share, lengths
        self.c, _, table = _cache(rng, lengths, [Q] * len(lengths), 16, 2, 128, garbage=False)
        self.bounds = S.SamBounds(self.c)
        self.q = [torch.from_numpy(rng.standard_normal((len(lengths), Q, H, 128))).to(DEV, torch.bfloat16) for _ in range(4)]
        self.lists = [_i32(_lists(rng, lengths, [Q] * len(lengths), Q, 2, 16, share, 9, table.shape[1])) for _ in range(4)]

    def run(self, i, q=None, lists=None):
        """Bounds of layer i from nothing, blocks of it, and attention over them and over lists that were there."""
        layer, q, lists = i & 1, self.q[i] if q is None else q, self.lists[i] if lists is None else lists
        self.bounds.codes[:, layer].zero_()
        self.bounds.exps[:, layer].zero_()
        self.bounds.update(layer, self.Q)
        blocks = self.bounds.select(layer, q, 9, share=self.share)
        return (blocks, *self.c.attend_blocks(layer, q, blocks, share=self.share), *self.c.attend_blocks(layer, q, lists, share=self.share))

    def apart(self):
        out = []
        for i in range(4):
            torch.cuda.synchronize()
            out.append([x.clone() for x in self.run(i)])
            torch.cuda.synchronize()
        return out


def _same(got, want):
    return all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("shape", SHAPES)
def test_one_call_after_the_other(shape):
    s = Calls(*shape)
    wants = s.apart()
    for _ in range(20):
        gots = [s.run(i) for i in range(4)]
        assert all(_same(g, w) for g, w in zip(gots, wants))
    assert s.c.status()[1] == 0


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("behind", ["nothing", "fill", "stream", "two streams"])
def test_recorded_behind(shape, behind):
    """The recorded call's first kernel is the selection's or the attention's, whatever it follows."""
    s = Calls(*shape)
    wants = s.apart()
    q, lists = s.q[0].clone(), s.lists[0].clone()
    src_q, src_l = q.clone(), lists.clone()
    for what in ("select", "attend"):
        def call():
            if what == "select":
                return (s.bounds.select(0, q, 9, share=s.share),)
            return s.c.attend_blocks(0, q, lists, share=s.share)
        s.bounds.update(0, s.Q)
        s.run(0)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            main = torch.cuda.current_stream()
            if behind == "fill":
                q.zero_()
                q.copy_(src_q)
            elif behind != "nothing":
                sides = [torch.cuda.Stream() for _ in range(1 if behind == "stream" else 2)]
                for side, to, frm in zip(sides, (q, lists), (src_q, src_l)):
                    side.wait_stream(main)
                    with torch.cuda.stream(side):
                        to.copy_(frm)
                s.lists[3].add_(0)                         # a kernel of the main stream's own
                for side in sides:
                    main.wait_stream(side)
            got = call()
        for i in (0, 2, 0):
            if behind == "nothing":
                q.copy_(s.q[i])
                lists.copy_(s.lists[i])
            else:
                src_q.copy_(s.q[i])
                src_l.copy_(s.lists[i])
                if behind != "two streams":
                    lists.copy_(s.lists[i])
            for _ in range(3):
                g.replay()
            want = (wants[i][0],) if what == "select" else wants[i][3:]
            assert _same(got, want), (what, i)
    assert s.c.status()[1] == 0


def test_two_threads_of_one_stream():
    """What one host thread starts may come between the two kernels of another's call."""
    import threading
    a, b = Calls(*SHAPES[1], seed=1), Calls(*SHAPES[1], seed=2)
    want = [a.apart(), b.apart()]
    torch.cuda.synchronize()
    got = [[], []]

    def work(k, s):
        for _ in range(10):
            got[k].append([s.run(i) for i in range(4)])
    threads = [threading.Thread(target=work, args=x) for x in enumerate((a, b))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for k in range(2):
        assert len(got[k]) == 10 and all(_same(g, w) for calls in got[k] for g, w in zip(calls, want[k]))


@pytest.mark.parametrize("B,K,V,masks", [(1, 1, 5, False), (4, 3, 50257, True), (40, 16, 9000, False), (7, 8, 151936, True)])
@pytest.mark.parametrize("how", ["calls", "recorded", "recorded behind a stream"])
def test_shaped_choices(B, K, V, masks, how):
    """Keys that hold anything before, logits and drafts that were written just before, drafts that change between the two calls."""
    gen = torch.Generator(device=DEV).manual_seed(B + V)
    logits = torch.empty(B, K + 1, V, dtype=torch.bfloat16, device=DEV)
    src = [torch.randn(B, K + 1, V, generator=gen, device=DEV).bfloat16() for _ in range(3)]
    words = -(-V // 32)
    mask = torch.randint(-(1 << 31), 1 << 31, (3, words), generator=gen, dtype=torch.int64, device=DEV).int() if masks else None
    mask_of = torch.randint(-1, 3, (B, K + 1), generator=gen, device=DEV).int() if masks else None
    shape = S.SamShape(V, masks=mask, mask_of=mask_of)
    keys = torch.empty(B * (K + 1), dtype=torch.int64, device=DEV)
    drafts, out = torch.zeros(B, K, dtype=torch.int32, device=DEV), torch.zeros(B, K + 1, dtype=torch.int32, device=DEV)
    accepted, n = torch.zeros_like(out), torch.zeros(B, dtype=torch.int32, device=DEV)
    values = torch.zeros(B, K + 1, device=DEV)
    n_draft = torch.full((B,), K, dtype=torch.int32, device=DEV)
    # what it comes to: rows without penalties are the first largest of what is allowed
    wants = []
    for x in src:
        y = x.float()
        if masks:
            bits = (mask[:, :, None] >> torch.arange(32, device=DEV)) & 1
            allowed = bits.flatten(1)[:, :V].bool()
            allowed = torch.cat([allowed, torch.ones(1, V, dtype=torch.bool, device=DEV)])[torch.where(mask_of < 0, 3, mask_of).long()]
            y = torch.where(allowed, y, -float("inf"))
        top = y.amax(-1)
        wants.append((torch.where(y == top[..., None], torch.arange(V, device=DEV), V).amin(-1).int(), top))
    now = src[0].clone()

    def call():
        keys.fill_(-1)
        logits.copy_(now)
        drafts.fill_(7)
        S.sam_argmax_shaped(logits, V, B, K, V, drafts, shape, keys)
        drafts.copy_(chosen)
        S.sam_verify_from_keys(keys, B, K, drafts, n_draft, out, accepted, n, values=values)

    chosen = wants[0][0][:, :K].clone()
    call()
    torch.cuda.synchronize()
    if how != "calls":
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            if how != "recorded":
                main, side = torch.cuda.current_stream(), torch.cuda.Stream()
                side.wait_stream(main)
                with torch.cuda.stream(side):
                    values.fill_(3)
                n.fill_(9)
                main.wait_stream(side)
            call()
    for i in (0, 1, 2, 1, 0, 2) * 3:
        now.copy_(src[i])
        chosen.copy_(wants[i][0][:, :K])
        if i == 2:
            chosen[:, -1] += 1
        call() if how == "calls" else g.replay()
        argmax, top = wants[i]
        assert torch.equal(out, argmax) and torch.equal(values, top)
        assert (n == (K if i == 2 else K + 1)).all()
