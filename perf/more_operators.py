"""Cases of four operators around the paged 4-bit cache and the verification of drafts: queries and keys rotated on their
way into the cache, blocks of the context selected by a cheap score, attention over the selected blocks, and verification of
logits under penalties, biases and grammar masks.

``listed()`` and ``draw()`` give cases, ``prepare()`` makes the tensors that a serving program holds before the call,
``run()`` makes one pass - the plain torch form where ``own`` is false, the package's calls where it is true -
``exact()`` states the result in 64 bits, and ``work()`` counts what the pass cannot do without.

Format of the cache: 16 neighbouring channels of one token and head share an e4m3 scale; a value is
``code * scale * 2**exp`` with an e2m1 code.  A tile holds 16 tokens of one head: key codes [16, D/2], value codes
[16, D/2], key scales [16, D/16], value scales [16, D/16] (low nibble = even channel).  A page holds the tiles
[layer, head, page_tokens / 16] of its tokens.  The bounds of a page are, for each layer and head, the largest and the
smallest key of every channel as 8-bit codes with one power of two.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
K_EXP, V_EXP = 0, -3            # exponents of the two halves of the cache
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    def rotate(name, B, Q, H, Hkv, D, tokens, P, dtype, R=0, interleaved=False, base=10000.0, layers=1, ragged=True):
        return dict(name=name, op="rotate", B=B, Q=Q, H=H, Hkv=Hkv, D=D, tokens=tokens, P=P, dtype=dtype, R=R or D,
                    interleaved=interleaved, base=base, layers=layers, ragged=ragged)

    def blocks(name, op, B, Q, H, Hkv, D, tokens, P, dtype, n_blocks, share=1, n_sink=1, n_recent=2, layers=1,
               ragged=True):
        return dict(name=name, op=op, B=B, Q=Q, H=H, Hkv=Hkv, D=D, tokens=tokens, P=P, dtype=dtype, n_blocks=n_blocks,
                    share=share, n_sink=n_sink, n_recent=n_recent, layers=layers, ragged=ragged)

    def shaped(name, B, K, V, said, n_bias, masks, free):
        return dict(name=name, op="shaped", B=B, K=K, V=V, said=said, n_bias=n_bias, masks=masks, free=free)

    return [
        # the proposals of a full batch, contexts of every length
        rotate("rotate_verify", 256, 17, 32, 8, 128, 300, 16, "bf16", layers=2),
        # a chunk of a long prompt, half of the channels rotated in neighbouring pairs, far positions
        rotate("rotate_prompt", 1, 20000, 28, 4, 128, 150003, 64, "fp16", R=64, interleaved=True, base=1e6, ragged=False),
        # a serving batch without proposals: which 64 of up to 2,048 pages each key head reads
        blocks("select_batch", "select", 64, 1, 32, 8, 128, 32768, 16, "bf16", 64),
        # proposals of sixteen share one selection a stream and key head
        blocks("select_verify", "select", 48, 17, 28, 4, 128, 12000, 16, "bf16", 96, share=17),
        # a chunk of a prompt, a selection for each query
        blocks("select_prompt", "select", 1, 1024, 28, 4, 128, 60011, 64, "fp16", 32, ragged=False),
        # one stream, one token: the launch is what counts
        blocks("blocks_token", "blocks", 1, 1, 32, 8, 128, 5000, 16, "bf16", 32, layers=2),
        # the serving batch over 1,024 selected tokens
        blocks("blocks_batch", "blocks", 64, 1, 32, 8, 128, 32768, 16, "bf16", 64),
        # proposals of sixteen over 2,048 tokens that they share
        blocks("blocks_verify", "blocks", 48, 17, 64, 8, 128, 20000, 32, "fp16", 64, share=17),
        # a chunk of a prompt, every sixteen queries over 2,048 tokens of their own
        blocks("blocks_prompt", "blocks", 1, 2048, 28, 4, 64, 60011, 64, "bf16", 32, share=16, ragged=False),
        # four agents, proposals of three, penalties and no grammar
        shaped("shaped_small", 4, 3, 151936, 1500, 8, 0, 0.0),
        # a full batch with long histories, every stream with its own penalties and biases
        shaped("shaped_batch", 192, 16, 151936, 6000, 64, 0, 0.0),
        # the same under grammars: half of the masks leave nearly all tokens, half of them a few hundred
        shaped("shaped_grammar", 128, 8, 151936, 2000, 16, 300, 0.5),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))

    op = rng.choice(("rotate", "select", "blocks", "blocks", "shaped"))
    if op == "shaped":
        K = rng.choice((1, 3, 4, 8, 16))
        V = rng.choice((151936, 32000, 128256, log_int(1000, 200000)))
        B = log_int(1, max(1, min(256, 192 * 17 * 151936 // ((K + 1) * V))))
        masks = rng.choice((0, log_int(1, 400)))
        return dict(op=op, B=B, K=K, V=V, said=log_int(1, 8000), n_bias=rng.choice((0, log_int(1, 300))), masks=masks,
                    free=rng.choice((0.0, 0.5, 1.0)) if masks else 0.0)
    dtype = rng.choice(("bf16", "fp16"))
    P = rng.choice((16, 16, 32, 64, 128))
    D = rng.choice((64, 128, 128))
    Hkv = rng.choice((1, 2, 4, 8))
    g = rng.choice((1, 2, 3, 4, 5, 7, 8))
    if op == "rotate":
        Q = rng.choice((1, 17, log_int(2, 33), log_int(34, min(20000, 20000 * 36 * 128 // (Hkv * (g + 2) * D)))))
        B = log_int(1, max(1, min(512, 20000 * 36 * 128 // (Q * Hkv * (g + 2) * D))))
        return dict(op=op, B=B, Q=Q, H=Hkv * g, Hkv=Hkv, D=D, tokens=log_int(1, 250000 if B < 16 else 2000), P=P,
                    dtype=dtype, R=rng.choice((D, D, D // 2, 32)), interleaved=rng.random() < 0.4,
                    base=rng.choice((1e4, 5e5, 1e6)), layers=rng.choice((1, 2)), ragged=rng.random() < 0.7)
    share = rng.choice((1, 1, log_int(2, 17), 16))
    Q = rng.choice((1, share, log_int(1, 33), log_int(34, 1000)))
    B = log_int(1, 64) if Q <= 33 else 1
    lists = B * -(-Q // share)
    room = min(64 * 32768 * 8 * 128 // (B * Hkv * D), 1024 * 28 * 60011 * P // (B * Q * Hkv * g * 64))
    tokens = log_int(1, max(2, min(120000, room)))
    n_sink, n_recent = rng.choice((0, 1, 1, 2)), rng.choice((1, 2, 3))
    least = n_sink + n_recent + -(-(share + P - 2) // P)
    most = 128 * 32 * 64 * 4 * 64 // (lists * Hkv * P * D)
    return dict(op=op, B=B, Q=Q, H=Hkv * g, Hkv=Hkv, D=D, tokens=tokens, P=P, dtype=dtype,
                n_blocks=max(least, min(log_int(4, 128), most)), share=share, n_sink=n_sink, n_recent=n_recent,
                layers=rng.choice((1, 2)), ragged=rng.random() < 0.7)


def _lengths(case):
    """Context lengths of the streams before this pass; the same set for every seed."""
    n, t = case["B"], case["tokens"]
    if not case["ragged"]:
        return [max(0, t - i) for i in range(n)]
    return [int(t * (0.1 + 0.9 * (0.6180339887498949 * i % 1.0))) if i else t for i in range(n)]


def _counts(case):
    """New tokens of the streams: full proposals and shorter ones."""
    n, Q = case["B"], case["Q"]
    if not case["ragged"]:
        return [Q] * n
    return [Q - (i * 5) % ((Q + 1) // 2 + 1) if i else Q for i in range(n)]


# ------------------------------------------------------------------------------------------------ the format, plainly
def _quantise(x, exp):
    """float32 [..., D] -> (codes uint8 [..., D], scale bytes uint8 [..., D/16])."""
    b = x.unflatten(-1, (-1, 16)) * 2.0 ** -exp
    s = (b.abs().amax(-1) / 6).clamp(max=448.0).to(torch.float8_e4m3fn)
    y = b.abs() / s.float()[..., None]
    code = torch.zeros_like(y, dtype=torch.uint8)
    for t, even in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)):
        code += (y >= t) if even else (y > t)
    code += b.signbit().to(torch.uint8) * 8
    code *= (s.float() > 0)[..., None]
    return code.flatten(-2), s.view(torch.uint8)


def _nibbles(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


def _split(tiles, D):
    """Bytes [..., 18 D] of tiles -> key codes, value codes [..., 16, D/2], key scales, value scales [..., 16, D/16]."""
    a, b, c = 8 * D, 16 * D, 17 * D
    return (tiles[..., :a].unflatten(-1, (16, D // 2)), tiles[..., a:b].unflatten(-1, (16, D // 2)),
            tiles[..., b:c].unflatten(-1, (16, D // 16)), tiles[..., c:].unflatten(-1, (16, D // 16)))


def _values(codes, scales, exp):
    """Packed codes [..., D/2] and scale bytes [..., D/16] -> float32 [..., D]."""
    half = torch.tensor(E2M1, device=codes.device)
    lut = torch.cat([half, -half])
    both = torch.stack([lut.repeat(16), lut.repeat_interleave(16)], 1)   # byte -> (even channel, odd channel)
    v = both[codes.int()].flatten(-2)
    s = scales.contiguous().view(torch.float8_e4m3fn).float() * 2.0 ** exp
    return (v.unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2)


def _exponent(amax):
    """The least power of two e for which amax <= 127 * 2**e, within 2**-6 of amax; 0 where amax is 0."""
    m, x = torch.frexp(amax)
    return torch.where(amax > 0, x - 6 - (m <= 127 / 128).int(), 0)


def _pow2(e):
    return torch.ldexp(torch.ones(e.shape, device=e.device), e)


def _bounds_of(tiles, D):
    """Tiles [..., P/16, 18 D] of pages -> codes int8 [..., 2, D] (largest up, smallest down), exponents int8 [...]."""
    kc, _, ks, _ = _split(tiles, D)
    k = _values(kc, ks, K_EXP).flatten(-3, -2)
    hi, lo = k.amax(-2), k.amin(-2)
    e = _exponent(torch.maximum(hi.abs(), lo.abs()).amax(-1))
    down = _pow2(-e)[..., None]
    return torch.stack([(hi * down).ceil(), (lo * down).floor()], -2).to(torch.int8), e.to(torch.int8)


# ------------------------------------------------------------------------------------------------ states
def _pool(case, n_pages, gen):
    """Pages of normally distributed keys (channels of unequal size) and values."""
    L, Hkv, P, D = case["layers"], case["Hkv"], case["P"], case["D"]
    pages = torch.empty(n_pages, L, Hkv, P // 16, 18 * D, dtype=torch.uint8, device=DEV)
    size = torch.exp(0.4 * torch.randn(L, Hkv, 1, 1, D, generator=gen, device=DEV))
    step = max(1, (1 << 26) // (L * Hkv * P * D))
    for at in range(0, n_pages, step):
        kc, vc, ks, vs = _split(pages[at:at + step], D)
        shape = kc.shape[:-1] + (D,)
        # what the tokens of a page have in common is what makes pages differ
        topic = torch.randn(shape[:-3] + (1, 1, D), generator=gen, device=DEV)
        for c, s, exp, mul, add in ((kc, ks, K_EXP, size, topic), (vc, vs, V_EXP, 0.5, 0.0)):
            code, scale = _quantise(torch.randn(shape, generator=gen, device=DEV) * mul + add, exp)
            c.copy_(_nibbles(code))
            s.copy_(scale)
    return pages


def _book(state, case, lengths, gen):
    """Tables over pages in no order, room for the new tokens; what is left is free."""
    B, P, Q = case["B"], case["P"], case["Q"]
    held = -(-(lengths + Q) // P)
    n_pages, max_pages = int(held.sum()) + 3, int(held.max())
    order = torch.randperm(n_pages, generator=gen, device=DEV).int()
    first = torch.cumsum(held, 0) - held
    at = torch.arange(max_pages, device=DEV)[None]
    has = at < held[:, None]
    table = torch.where(has, order[(first[:, None] + at).clamp(max=n_pages - 1)], -1)
    ref = torch.zeros(n_pages, dtype=torch.int32, device=DEV)
    ref[table[has].long()] = 1
    free = torch.zeros_like(ref)
    free[:3] = order[n_pages - 3:]
    state["book"] = dict(page_table=table.contiguous(), seq_len=lengths.int(), ref_count=ref, free_list=free,
                         meta=torch.tensor([3, 0, 0, 0], dtype=torch.int32, device=DEV))
    return n_pages


def _complete(case, seq, new):
    """[B, n] places in the table, and whether the page there is filled up by the new tokens."""
    P = case["P"]
    at = seq[:, None] // P + torch.arange(case["Q"] // P + 1, device=DEV)
    return at, at < ((seq + new.clamp(min=0)) // P)[:, None]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    state = dict(case=case)
    if case["op"] == "shaped":
        _prepare_shaped(state, case, gen)
        return state
    B, Q, H, Hkv, D, P = (case[x] for x in ("B", "Q", "H", "Hkv", "D", "P"))
    seq = torch.tensor(_lengths(case), device=DEV)[torch.randperm(B, generator=gen, device=DEV)]
    new = torch.tensor(_counts(case), dtype=torch.int32, device=DEV)[torch.randperm(B, generator=gen, device=DEV)]
    state["n_new"], state["layer"] = new, case["layers"] - 1
    n_pages = _book(state, case, seq, gen)
    state["pages"] = _pool(case, n_pages, gen)
    # queries, keys and values are slices of the projection's output
    qkv = torch.randn(B, Q, H + 2 * Hkv, D, generator=gen, device=DEV)
    qkv[:, :, H + Hkv:] *= 0.5
    state["qkv"] = qkv.to(TYPES[case["dtype"]])
    if case["op"] == "rotate":
        state["inv_freq"] = [case["base"] ** (-2 * i / case["R"]) for i in range(case["R"] // 2)]
    elif case["op"] == "select":
        codes = torch.empty(n_pages, case["layers"], Hkv, 2, D, dtype=torch.int8, device=DEV)
        exps = torch.empty(n_pages, case["layers"], Hkv, dtype=torch.int8, device=DEV)
        step = max(1, (1 << 26) // (case["layers"] * Hkv * P * D))
        for a in range(0, n_pages, step):
            codes[a:a + step], exps[a:a + step] = _bounds_of(state["pages"][a:a + step], D)
        at, full = _complete(case, seq, new)
        gone = state["book"]["page_table"].gather(1, at.clamp(max=state["book"]["page_table"].shape[1] - 1))[full].long()
        codes[gone, state["layer"]], exps[gone, state["layer"]] = 0, 0       # this pass has to make these
        state["codes"], state["exps"] = codes, exps
    else:
        # lists as a selection leaves them: the first page, the last ones, others in between, in order
        share, n = case["share"], case["n_blocks"]
        lists = -(-Q // share)
        first = seq[:, None] + torch.arange(lists, device=DEV) * share            # [B, lists]
        last = torch.minimum(first + share, (seq + new)[:, None]) - 1
        at = torch.arange(state["book"]["page_table"].shape[1], device=DEV)
        rank = torch.rand(B, lists, Hkv, at.numel(), generator=gen, device=DEV)
        must = (at < case["n_sink"]) | (at > (first // P - case["n_recent"])[..., None])
        rank = rank.add_(must[:, :, None] * 1.0)
        rank.masked_fill_((at > (last // P)[..., None])[:, :, None] | (last < first)[..., None, None], -1.0)
        top = rank.topk(min(n, at.numel()), -1)
        b = torch.where(top.values >= 0, top.indices, 1 << 30).sort(-1).values.int()
        b = torch.nn.functional.pad(b, (0, n - b.shape[-1]), value=1 << 30)
        state["blocks"] = torch.where(b < 1 << 30, b, -1).contiguous()
    if own:
        _handles(state, case)
    return state


def _handles(state, case):
    """What a program that uses the package keeps: the cache object over the tensors, the rotation, the bounds."""
    import paper_2512_18337_b200 as S
    b = state["book"]
    c = state["cache"] = S.SamCache(n_pages=b["ref_count"].numel(), page_tokens=case["P"], n_streams=case["B"],
                                    max_pages=b["page_table"].shape[1], n_layers=case["layers"], n_kv_heads=case["Hkv"],
                                    head_dim=case["D"], k_exp=K_EXP, v_exp=V_EXP, device=DEV,
                                    tensors=dict(pages=state["pages"], **b))
    if case["op"] == "rotate":
        state["rope"] = S.SamRope(state["inv_freq"], interleaved=case["interleaved"], device=DEV)
    elif case["op"] == "select":
        state["bounds"] = S.SamBounds(c, codes=state["codes"], exps=state["exps"])


def _prepare_shaped(state, case, gen):
    B, K, V, said = case["B"], case["K"], case["V"], case["said"]
    state["logits"] = torch.empty(B * (K + 1), V, dtype=torch.bfloat16, device=DEV)
    state["logits"].normal_(generator=gen).mul_(2.0)
    rows = state["logits"].view(B, K + 1, V)
    # what was said: a few tokens often, many once; half of it was the prompt
    zipf = torch.rand(B, said, generator=gen, device=DEV).pow_(4).mul_(V).long().clamp_(max=V - 1)
    half = said // 2
    counts = torch.zeros(B, V, dtype=torch.int32, device=DEV)
    counts.scatter_add_(1, zipf[:, half:], torch.ones_like(zipf[:, half:], dtype=torch.int32))
    told = torch.zeros(B, V, dtype=torch.bool, device=DEV)
    told.scatter_(1, zipf[:, :half], True)
    state["counts"] = torch.where(told, counts | -(1 << 31), counts)
    state["seen"] = _bits(state["counts"] != 0)
    # the model wants to go on, and to repeat itself
    drafts = torch.randint(V, (B, K), generator=gen, device=DEV)
    again = torch.rand(B, K, generator=gen, device=DEV) < 0.3
    pick = zipf[torch.arange(B, device=DEV)[:, None], torch.randint(said, (B, K), generator=gen, device=DEV)]
    state["drafts"] = torch.where(again, pick, drafts).int()
    top = rows.amax(-1).float()
    liked = torch.rand(B, K, generator=gen, device=DEV) < 0.7
    at = state["drafts"].long()[..., None]
    old = rows[:, :K].gather(2, at)
    rows[:, :K].scatter_(2, at, torch.where(liked[..., None], (top[:, :K, None] + 1.5).bfloat16(), old))
    often = zipf[:, :1, None].expand(B, K + 1, 1)
    rows.scatter_(2, often, (top[..., None] + 1.0).bfloat16())
    state["n_draft"] = torch.randint(0, K + 1, (B,), generator=gen, device=DEV).int()
    u = torch.rand(3, B, generator=gen, device=DEV)
    state["repetition"], state["presence"], state["frequency"] = 1 + 0.3 * u[0], 0.7 * u[1], 0.4 * u[2]
    n = case["n_bias"]
    state["bias_tokens"] = torch.randint(V, (B, n), generator=gen, device=DEV).int()
    state["bias_values"] = torch.randn(B, n, generator=gen, device=DEV) * 4
    state["n_bias"] = torch.randint(0, n + 1, (B,), generator=gen, device=DEV).int()
    state["masks"] = state["mask_of"] = None
    if case["masks"]:
        m, few = case["masks"], round(case["masks"] * (1 - case["free"]))
        share = torch.full((m, 1), 0.97, device=DEV)
        share[:few] = min(1.0, 300 / V)
        state["masks"] = torch.cat([_bits(torch.rand(1, V, generator=gen, device=DEV) < share[i:i + 1]) for i in range(m)])
        state["mask_of"] = torch.randint(-1, m, (B, K + 1), generator=gen, device=DEV).int()
    state["argmax"] = torch.empty(B, K + 1, dtype=torch.int32, device=DEV)
    state["accepted"], state["n_accepted"] = torch.empty_like(state["argmax"]), torch.empty_like(state["n_draft"])
    state["values"] = torch.empty(B, K + 1, device=DEV)
    state["keys"] = torch.zeros(B * (K + 1), dtype=torch.int64, device=DEV)
    if own:
        import paper_2512_18337_b200 as S
        state["shape"] = S.SamShape(
            V, counts=state["counts"], seen=state["seen"], repetition=state["repetition"], presence=state["presence"],
            frequency=state["frequency"], bias_tokens=state["bias_tokens"], bias_values=state["bias_values"],
            n_bias=state["n_bias"], masks=state["masks"], mask_of=state["mask_of"])


def _bits(x):
    """bool [n, V] -> int32 [n, ceil(V / 32)], token t in bit t % 32 of word t / 32."""
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % 32)).view(x.shape[0], -1, 32)
    w = (x.long() << torch.arange(32, device=x.device)).sum(-1)
    return torch.where(w < 1 << 31, w, w - (1 << 32)).int()


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    return dict(rotate=_rotate, select=_select, blocks=_blocks, shaped=_shaped)[state["case"]["op"]](state)


def _rotate(state):
    """Queries and keys rotated to their positions, keys and values into the cache and back as later steps see them."""
    case, book = state["case"], state["book"]
    H, Hkv, Q = case["H"], case["Hkv"], case["Q"]
    q, k, v = state["qkv"][:, :, :H], state["qkv"][:, :, H:H + Hkv], state["qkv"][:, :, H + Hkv:]
    if own:
        c = state["cache"]
        y = c.append_rotated(state["layer"], q, k, v, state["rope"], n_new=state["n_new"])
        return (y, *c.read(state["layer"], first=book["seq_len"], n=state["n_new"], max_n=Q, dtype=k.dtype))
    return _rotate_plain(state, q, k, v)


def _rotate_plain(state, q, k, v):
    case, book = state["case"], state["book"]
    Q, P, D, R = case["Q"], case["P"], case["D"], case["R"]
    i = torch.arange(Q, device=DEV)
    pos = book["seq_len"][:, None].long() + i                                     # [B, Q]
    angle = pos[..., None].double() * torch.tensor(state["inv_freq"], dtype=torch.float64, device=DEV)
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    used = i < state["n_new"][:, None]

    def turn(x):
        y = x.float()
        a, b = (y[..., 0:R:2], y[..., 1:R:2]) if case["interleaved"] else (y[..., :R // 2], y[..., R // 2:R])
        c, d = a * cos - b * sin, b * cos + a * sin
        z = torch.stack([c, d], -1).flatten(-2) if case["interleaved"] else torch.cat([c, d], -1)
        return torch.cat([z, y[..., R:]], -1)

    page = book["page_table"].gather(1, pos // P)
    on = used & (page >= 0)
    kc, vc, ks, vs = _split(state["pages"][:, state["layer"]], D)                 # [pages, Hkv, P/16, 16, ...]
    at = (page[on].long(), slice(None), pos[on] % P // 16, pos[on] % 16)
    out = [torch.where(used[..., None, None], turn(q), 0.0).to(q.dtype)]
    for x, codes, scales, exp in ((turn(k), kc, ks, K_EXP), (v.float(), vc, vs, V_EXP)):
        code, scale = _quantise(x[on], exp)
        codes[at] = _nibbles(code)
        scales[at] = scale
        y = torch.zeros(x.shape, dtype=k.dtype, device=DEV)
        y[on] = _values(codes[at], scales[at], exp).to(k.dtype)
        out.append(y)
    return tuple(out)


def _select(state):
    """Bounds of the pages that the new tokens fill up, then the blocks that each list of queries will read."""
    case, q = state["case"], state["qkv"][:, :, :state["case"]["H"]]
    if own:
        b = state["bounds"]
        b.update(state["layer"], case["Q"], n_new=state["n_new"])
        blocks = b.select(state["layer"], q, case["n_blocks"], n_sink=case["n_sink"], n_recent=case["n_recent"],
                          share=case["share"], n_new=state["n_new"])
    else:
        blocks = _select_plain(state, q)
    return blocks, state["codes"], state["exps"]


def _select_plain(state, q):
    case, book, layer = state["case"], state["book"], state["layer"]
    B, Q, H, Hkv, D, P, n, share = (case[x] for x in ("B", "Q", "H", "Hkv", "D", "P", "n_blocks", "share"))
    seq, new, table = book["seq_len"].long(), state["n_new"], book["page_table"]
    at, full = _complete(case, seq, new)
    page = table.gather(1, at.clamp(max=table.shape[1] - 1))[full].long()
    state["codes"][page, layer], state["exps"][page, layer] = _bounds_of(state["pages"][page, layer], D)
    # queries in eight bits
    x = q.float()
    e = _exponent(x.abs().amax(-1))
    x = torch.round(x * _pow2(-e)[..., None])
    lists, g = -(-Q // share), H // Hkv
    pad = lists * share - Q
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, pad)).view(B, lists, share, Hkv, g, D).permute(0, 3, 1, 2, 4, 5)
    e = torch.nn.functional.pad(e, (0, 0, 0, pad)).view(B, lists, share, Hkv, g).permute(0, 3, 1, 2, 4)
    x = torch.cat([x.clamp(min=0), x.clamp(max=0)], -1).reshape(B, Hkv, -1, 2 * D)
    c = state["codes"][:, layer][table.clamp(min=0).long()].transpose(1, 2).flatten(-2).float()   # [B, Hkv, M, 2 D]
    ce = state["exps"][:, layer][table.clamp(min=0).long()].transpose(1, 2).int()                 # [B, Hkv, M]
    best = torch.empty(B, lists, Hkv, table.shape[1], device=DEV)
    step = max(1, (1 << 28) // (B * Hkv * share * g * table.shape[1]))
    for a in range(0, lists, step):
        z = min(lists, a + step)
        s = torch.matmul(x[:, :, a * share * g:z * share * g], c.transpose(-1, -2))               # exact: whole numbers
        s = s.view(B, Hkv, z - a, share * g, -1) * _pow2(e[:, :, a:z].flatten(-2))[..., None]
        i = torch.arange(a * share, z * share, device=DEV).view(z - a, share, 1).expand(-1, -1, g).flatten(1)
        s.masked_fill_((i >= new[:, None, None])[:, None, ..., None], -math.inf)
        best[:, a:z] = (s.amax(-2) * _pow2(ce)[:, :, None]).transpose(1, 2)
    first = seq[:, None] + torch.arange(lists, device=DEV) * share
    last = torch.minimum(first + share, (seq + new)[:, None]) - 1
    m = torch.arange(table.shape[1], device=DEV)
    must = (m < case["n_sink"]) | (m > (first // P - case["n_recent"])[..., None])
    best.masked_fill_(must[:, :, None], math.inf)
    on = (m <= (last // P)[..., None]) & (last >= first)[..., None] & (table >= 0)[:, None]
    best.masked_fill_(~on[:, :, None], -math.inf)
    pick = torch.sort(best, dim=-1, descending=True, stable=True)
    got = torch.where(pick.values > -math.inf, pick.indices, 1 << 30)[..., :n].sort(-1).values
    got = torch.nn.functional.pad(got, (0, n - got.shape[-1]), value=1 << 30)
    return torch.where(got < 1 << 30, got, -1).int()


def _blocks(state):
    """Attention of the new rows over the blocks of their lists; their keys and values are in the cache already."""
    case, q = state["case"], state["qkv"][:, :, :state["case"]["H"]]
    if own:
        return state["cache"].attend_blocks(state["layer"], q, state["blocks"], share=case["share"], n_new=state["n_new"])
    return _blocks_plain(state, q)


def _blocks_plain(state, q):
    case, book = state["case"], state["book"]
    B, Q, H, Hkv, D, P, n, share = (case[x] for x in ("B", "Q", "H", "Hkv", "D", "P", "n_blocks", "share"))
    lists, g = -(-Q // share), H // Hkv
    pages, table = state["pages"][:, state["layer"]], book["page_table"]
    out = torch.zeros(B, lists * share, H, D, device=DEV)
    lse = torch.full((B, lists * share, H), -math.inf, device=DEV)
    x = torch.nn.functional.pad(q.float(), (0, 0, 0, 0, 0, lists * share - Q))
    head = torch.arange(Hkv, device=DEV)[:, None]
    step = max(1, (1 << 27) // (B * Hkv * n * P * D))
    for a in range(0, lists, step):
        z = min(lists, a + step)
        bl = state["blocks"][:, a:z].long()                                       # [B, l, Hkv, n]
        page = table[:, None, None].expand(-1, z - a, Hkv, -1).gather(3, bl.clamp(min=0))
        kc, vc, ks, vs = _split(pages[page.clamp(min=0).long(), head], D)         # [B, l, Hkv, n, P/16, 16, ...]
        tok = (bl[..., None] * P + torch.arange(P, device=DEV)).flatten(-2)       # [B, l, Hkv, n P]
        on = ((bl >= 0) & (page >= 0))[..., None].expand(-1, -1, -1, -1, P).flatten(-2)
        i = torch.arange(a * share, z * share, device=DEV).view(z - a, share)
        pos = book["seq_len"][:, None, None] + i                                  # [B, l, share]
        seen = on[:, :, :, None] & (tok[:, :, :, None] <= pos[:, :, None, :, None])
        seen &= (i < state["n_new"][:, None, None])[:, :, None, :, None]          # [B, l, Hkv, share, n P]
        y = x[:, a * share:z * share].view(B, z - a, share, Hkv, g, D).transpose(2, 3).flatten(3, 4)
        k = _values(kc, ks, K_EXP).flatten(3, 5)
        s = torch.matmul(y, k.transpose(-1, -2)).mul_(D ** -0.5).view(B, z - a, Hkv, share, g, -1)
        s.masked_fill_(~seen[:, :, :, :, None], -math.inf)
        m = s.amax(-1, keepdim=True)
        s.sub_(m.nan_to_num(neginf=0.0)).exp_()
        l = s.sum(-1, keepdim=True)
        o = torch.matmul(s.flatten(3, 4), _values(vc, vs, V_EXP).flatten(3, 5)).view(B, z - a, Hkv, share, g, D)
        o = torch.where(l > 0, o / l, 0.0).transpose(2, 3)
        out[:, a * share:z * share] = o.reshape(B, -1, H, D)
        lse[:, a * share:z * share] = (m + l.log()).squeeze(-1).transpose(2, 3).reshape(B, -1, H)
    return out[:, :Q].to(q.dtype).contiguous(), lse[:, :Q].contiguous()


def _shaped(state):
    """The greedy choice of every row under penalties, biases and masks, and what of each proposal it accepts."""
    case, s = state["case"], state
    B, K, V = case["B"], case["K"], case["V"]
    if own:
        import paper_2512_18337_b200 as S
        S.sam_argmax_shaped(s["logits"], V, B, K, V, s["drafts"], s["shape"], s["keys"])
        S.sam_verify_from_keys(s["keys"], B, K, s["drafts"], s["n_draft"], s["argmax"], s["accepted"], s["n_accepted"],
                               values=s["values"])
        return s["argmax"], s["accepted"], s["n_accepted"], s["values"]
    choice = torch.empty(B, K + 1, dtype=torch.int64, device=DEV)
    value = torch.empty(B, K + 1, device=DEV)
    step = max(1, (1 << 27) // ((K + 1) * V))
    for a in range(0, B, step):
        z = min(B, a + step)
        x = _shape_plain(s, slice(a, z), case)
        choice[a:z] = x.argmax(-1)
        value[a:z] = x.amax(-1)
    return *_accept_plain(choice, s, K), value


def _shape_plain(s, r, case):
    """Logits [b, K + 1, V] in 32 bits under penalties, biases and masks."""
    K, V = case["K"], case["V"]
    x = s["logits"].view(-1, K + 1, V)[r].float()
    # row j is asked after the drafts before it
    extra = torch.zeros(x.shape, dtype=torch.int32, device=DEV)
    d = s["drafts"][r].long()
    for j in range(1, K + 1):
        extra[:, j] = extra[:, j - 1]
        extra[:, j].scatter_add_(1, d[:, j - 1:j], torch.ones_like(d[:, :1], dtype=torch.int32))
    c = s["counts"][r][:, None]
    told, n = c < 0, (c & 0x7fffffff) + extra
    rep, pres, freq = (s[k][r][:, None, None] for k in ("repetition", "presence", "frequency"))
    x = torch.where(told | (n > 0), torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * n
    x = torch.where(n > 0, x - pres, x)
    if case["n_bias"]:
        at = torch.arange(case["n_bias"], device=DEV)
        y = torch.where(at < s["n_bias"][r][:, None], s["bias_values"][r], 0.0)
        bias = torch.zeros(x.shape[0], V, device=DEV)
        for i in range(case["n_bias"]):                                           # one after the other: the order counts
            bias.scatter_add_(1, s["bias_tokens"][r][:, i:i + 1].long(), y[:, i:i + 1])
        x = x + bias[:, None]
    if s["masks"] is not None:
        m = s["mask_of"][r].long()
        word = s["masks"][m.clamp(min=0)]
        bit = (word[..., None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        ok = bit.flatten(-2)[..., :V].bool() | (m < 0)[..., None]
        x = torch.where(ok, x, -math.inf)
    return x


def _accept_plain(choice, s, K):
    """Drafts are kept as long as they are the choice; then comes the choice itself."""
    j = torch.arange(K, device=DEV)
    same = (choice[:, :K] == s["drafts"]) & (j < s["n_draft"][:, None])
    a = same.int().cumprod(1).sum(1)
    j = torch.arange(K + 1, device=DEV)
    d = torch.nn.functional.pad(s["drafts"], (0, 1))
    acc = torch.where(j < a[:, None], d, torch.where(j == a[:, None], choice, -1))
    return choice.int(), acc.int(), (a + 1).int()


# ------------------------------------------------------------------------------------------------ in 64 bits
def _round_e2m1(y):
    """Nearest e2m1 value of a magnitude, ties to the even code."""
    q = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0)).double()
    return (torch.round(y / q) * q).clamp(max=6.0)


def _round_e4m3(v):
    q = torch.exp2(torch.floor(torch.log2(v.clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / q) * q).clamp(max=448.0)


def _in_four_bits(x, exp):
    x = x.unflatten(-1, (-1, 16))
    s = _round_e4m3(x.abs().amax(-1, keepdim=True) / (6 * 2.0 ** exp)) * 2.0 ** exp
    return torch.where(s > 0, x.sign() * _round_e2m1(x.abs() / s) * s, 0.0).flatten(-2)


def _read_exact(tiles, D, which):
    """Tiles [..., 18 D] -> their tokens [..., 16, D] in 64 bits, from the bit fields."""
    codes = tiles[..., which * 8 * D:(which + 1) * 8 * D].reshape(*tiles.shape[:-1], 16, D // 2)
    scales = tiles[..., (16 + which) * D:(17 + which) * D].reshape(*tiles.shape[:-1], 16, D // 16).double()
    nib = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).double()
    sign = 1 - 2 * torch.floor(nib / 8)
    e, f = torch.floor(nib % 8 / 2), nib % 2
    mag = torch.where(e > 0, (2 + f) * torch.exp2(e - 2), f / 2)
    se, sf = torch.floor(scales / 8), scales % 8
    s = torch.where(se > 0, (8 + sf) * torch.exp2(se - 10), sf * 2.0 ** -9)
    return sign * mag * s.repeat_interleave(16, -1) * 2.0 ** (V_EXP if which else K_EXP)


def exact(case, seed):
    state = prepare(case, seed)
    return dict(rotate=_rotate_exact, select=_select_exact, blocks=_blocks_exact, shaped=_shaped_exact)[case["op"]](state, case)


def _rotate_exact(state, case):
    Q, H, Hkv, R = case["Q"], case["H"], case["Hkv"], case["R"]
    x = state["qkv"].double()
    n, seq = state["n_new"].tolist(), state["book"]["seq_len"].tolist()
    f = torch.tensor(state["inv_freq"], dtype=torch.float64, device=DEV)
    for b in range(case["B"]):
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                           (seq[b] + torch.arange(Q, device=DEV).double())[:, None] * f)[:, None]
        y = x[b, :, :H + Hkv]
        re, im = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        z = torch.complex(y[..., re], y[..., im]) * turn
        y[..., re], y[..., im] = z.real, z.imag
        x[b, n[b]:] = 0
    return x[:, :, :H], _in_four_bits(x[:, :, H:H + Hkv], K_EXP), _in_four_bits(x[:, :, H + Hkv:], V_EXP)


def _whole(x):
    """Largest magnitudes -> the exponents of their 8-bit codes, by trying powers of two."""
    e = torch.zeros_like(x, dtype=torch.int64)
    for k in range(60, -61, -1):
        e = torch.where((x > 0) & (x <= 127 * 2.0 ** k), k, e)
    return e


def _select_exact(state, case):
    B, Q, H, Hkv, D, P, share = (case[x] for x in ("B", "Q", "H", "Hkv", "D", "P", "share"))
    if B * Hkv * -(-Q // share) > 6000:
        return None
    layer, g, lists = state["layer"], H // Hkv, -(-Q // share)
    seq, new = state["book"]["seq_len"].tolist(), state["n_new"].tolist()
    table = state["book"]["page_table"].tolist()
    codes, exps = state["codes"].clone(), state["exps"].clone()
    for b in range(B):
        for i in range(seq[b] // P, (seq[b] + new[b]) // P):
            k = _read_exact(state["pages"][table[b][i], layer], D, 0).flatten(1, 2)
            e = _whole(k.abs().amax((1, 2)))
            unit = torch.exp2(e.double())[:, None]
            codes[table[b][i], layer, :, 0] = torch.ceil(k.amax(1) / unit).to(torch.int8)
            codes[table[b][i], layer, :, 1] = torch.floor(k.amin(1) / unit).to(torch.int8)
            exps[table[b][i], layer] = e.to(torch.int8)
    out = torch.full((B, lists, Hkv, case["n_blocks"]), -1, dtype=torch.int32, device=DEV)
    for b in range(B):
        page = state["book"]["page_table"][b].long()
        for h in range(Hkv):
            hi, lo = codes[page, layer, h].long().unbind(1)
            unit = torch.exp2(exps[page, layer, h].double())
            q = state["qkv"][b, :, h * g:(h + 1) * g].double()
            u = torch.exp2(_whole(q.abs().amax(-1)).double())
            w = torch.round(q / u[..., None])
            # the larger of the two products of a channel: the one with the bound of the query's sign
            s = (torch.einsum("qgd,md->qgm", w.clamp(min=0), hi.double()) + torch.einsum("qgd,md->qgm", w.clamp(max=0), lo.double()))
            s = (s * u[..., None]).amax(1) * unit
            for l in range(lists):
                a, z = l * share, min((l + 1) * share, new[b])
                if z <= a:
                    continue
                n, old = (seq[b] + z - 1) // P + 1, (seq[b] + a) // P - case["n_recent"]
                t = s[a:z, :n].amax(0)
                t[:min(case["n_sink"], n)] = math.inf
                t[max(0, old + 1):] = math.inf
                keep = torch.argsort(t, descending=True, stable=True)[:case["n_blocks"]].sort().values
                out[b, l, h, :keep.numel()] = keep.int()
    return out, codes, exps


def _blocks_exact(state, case):
    B, Q, H, Hkv, D, P, share = (case[x] for x in ("B", "Q", "H", "Hkv", "D", "P", "share"))
    if B * Hkv * -(-Q // share) > 6000:
        return None
    g = H // Hkv
    seq, new = state["book"]["seq_len"].tolist(), state["n_new"].tolist()
    out = torch.zeros(B, Q, H, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, Q, H), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(B):
        for l in range(-(-Q // share)):
            a, z = l * share, min((l + 1) * share, new[b])
            if z <= a:
                continue
            pos = seq[b] + torch.arange(a, z, device=DEV)
            for h in range(Hkv):
                bl = state["blocks"][b, l, h]
                bl = bl[bl >= 0].long()
                tiles = state["pages"][state["book"]["page_table"][b][bl].long(), state["layer"], h]
                k, v = (_read_exact(tiles, D, w).reshape(-1, D) for w in (0, 1))
                t = (bl[:, None] * P + torch.arange(P, device=DEV)).flatten()
                x = state["qkv"][b, a:z, h * g:(h + 1) * g].double()
                s = torch.einsum("qgd,td->qgt", x, k) / math.sqrt(D)
                s = s.masked_fill((t > pos[:, None])[:, None], -math.inf)
                lse[b, a:z, h * g:(h + 1) * g] = torch.logsumexp(s, -1)
                out[b, a:z, h * g:(h + 1) * g] = torch.softmax(s, -1) @ v
    return out, lse


def _shaped_exact(state, case):
    B, K, V = case["B"], case["K"], case["V"]
    choice = torch.empty(B, K + 1, dtype=torch.int64, device=DEV)
    value = torch.empty(B, K + 1, dtype=torch.float64, device=DEV)
    n_bias = state["n_bias"].tolist()
    for b in range(B):
        said = (state["counts"][b].long() & 0x7fffffff).double()
        told = state["counts"][b] < 0
        bias = torch.zeros(V, dtype=torch.float64, device=DEV)
        bias.index_add_(0, state["bias_tokens"][b, :n_bias[b]].long(), state["bias_values"][b, :n_bias[b]].double())
        rep, pres, freq = (state[k][b].double() for k in ("repetition", "presence", "frequency"))
        for j in range(K + 1):
            if j:
                said[state["drafts"][b, j - 1].long()] += 1
            x = state["logits"][b * (K + 1) + j].double()
            x = torch.where(told | (said > 0), torch.where(x > 0, x / rep, x * rep), x)
            x = x - freq * said - pres * (said > 0) + bias
            if state["masks"] is not None and state["mask_of"][b, j] >= 0:
                w = state["masks"][state["mask_of"][b, j].long()].long()
                t = torch.arange(V, device=DEV)
                x = x.masked_fill((w[t // 32] >> (t % 32)) & 1 == 0, -math.inf)
            choice[b, j], value[b, j] = torch.argmax(x), x.max()
    return *_accept_plain(choice, state, K), value


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    if case["op"] == "shaped":
        B, K, V = case["B"], case["K"], case["V"]
        full, few = B * (K + 1), 0
        if case["masks"]:
            m = case["masks"]
            few = full * round(m * (1 - case["free"])) / (m + 1)
            full -= few
        words = 4 * -(-V // 32)
        # rows under a narrow mask need the logits of its tokens only
        bytes_ = full * 2 * V + few * 2 * min(300, V) + B * words + case["masks"] * words
        return {"bytes": bytes_ + B * (4 * min(case["said"], V) + 8 * case["n_bias"]) + B * (K + 1) * 8, "flops": 0}
    P, D, H, Hkv, Q = case["P"], case["D"], case["H"], case["Hkv"], case["Q"]
    lengths, counts = _lengths(case), _counts(case)
    if case["op"] == "rotate":
        n, every = sum(counts), len(counts) * Q
        # queries in and out, keys and values in 16 bits, into the cache, out of it, and in 16 bits again
        return {"bytes": n * (H + 2 * Hkv) * D * 2 + every * H * D * 2 + 2 * n * 2 * Hkv * D * 9 / 16 + every * 2 * Hkv * D * 2,
                "flops": 3 * n * (H + Hkv) * case["R"]}
    share, nb = case["share"], case["n_blocks"]
    lists = -(-Q // share)
    mean = sum(counts) / len(counts)
    used = sum(-(-c // share) for c in counts)
    if case["op"] == "select":
        pages = sum(l // P for l in lengths)
        full = sum(mean for l in lengths) / P
        return {"bytes": (pages + full) * Hkv * (2 * D + 1) + full * Hkv * P * D * 9 / 16 + sum(counts) * H * D * 2 +
                len(counts) * lists * Hkv * nb * 4, "flops": 4 * D * H * mean * pages}
    read = pairs = 0.0
    for l in lengths:                                       # lengths and counts meet in another order for each seed
        held = -(-(l + mean) // P)
        each = min(nb, held)
        # lists of one stream have pages in common
        read += min(held, each * used / len(counts)) * P
        pairs += mean * min(each * P, l + mean / 2)
    rows, out = sum(counts) * H, len(counts) * Q * H
    return {"bytes": read * Hkv * D * 9 / 8 + rows * D * 2 + out * (D * 2 + 4) + used * Hkv * nb * 4, "flops": 4 * D * H * pairs}
