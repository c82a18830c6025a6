"""Cases of the paged 4-bit key/value cache: attention over it, keys and values into and out of it, and its pages.

``listed()`` and ``draw()`` give cases, ``prepare()`` makes the tensors that a serving program holds before the call,
``run()`` makes one pass - the plain torch form where ``own`` is false, the package's calls where it is true -
``exact()`` states the result in 64 bits, and ``work()`` counts what the pass cannot do without.

Format of the cache: 16 neighbouring channels of one token and head share an e4m3 scale; a value is
``code * scale * 2**exp`` with an e2m1 code.  A tile holds 16 tokens of one head: key codes [16, D/2], value codes
[16, D/2], key scales [16, D/16], value scales [16, D/16] (low nibble = even channel).  A page holds the tiles
[layer, head, page_tokens / 16] of its tokens.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
K_EXP, V_EXP = 0, -3            # exponents of the two halves of the cache
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DROP = -(1 << 31)               # a count of kept tokens that empties a stream


# ------------------------------------------------------------------------------------------------ cases
def listed():
    def attend(name, B, Q, H, Hkv, D, tokens, P, dtype, ragged=True, window=0, layers=1):
        return dict(name=name, op="attend", B=B, Q=Q, H=H, Hkv=Hkv, D=D, tokens=tokens, P=P, dtype=dtype,
                    ragged=ragged, window=window, layers=layers)

    return [
        # one stream, one token, a short context: the launch is what counts
        attend("token_short", 1, 1, 32, 8, 128, 333, 16, "bf16", layers=2),
        # a serving batch without proposals, contexts of every length
        attend("token_batch", 64, 1, 32, 8, 128, 8191, 16, "bf16"),
        # one key head per query head, narrow heads, a sliding window over part of the context
        attend("token_window", 48, 1, 16, 16, 64, 6000, 32, "fp16", window=4000),
        # two agents with very long memories
        attend("token_long", 2, 1, 64, 8, 128, 250001, 64, "bf16", ragged=False),
        # the four-stream step with proposals of three
        attend("verify_small", 4, 4, 28, 4, 128, 2500, 16, "bf16"),
        # proposals of sixteen, some of them shorter, contexts of every length
        attend("verify_batch", 64, 17, 32, 8, 128, 12000, 16, "bf16"),
        # eight query heads to a key head
        attend("verify_wide", 16, 17, 64, 8, 128, 30000, 64, "fp16"),
        # a prompt taken in chunks: the last chunk attends to all that is in the cache
        attend("prompt_chunk", 1, 2048, 28, 4, 128, 20011, 16, "bf16", ragged=False),
        # keys and values of the proposals of a full batch
        dict(name="append_verify", op="append", B=256, Q=17, H=32, Hkv=8, D=128, tokens=300, P=16, dtype="bf16",
             ragged=True, layers=2),
        # a long prompt's keys and values, and what the cache makes of them
        dict(name="append_prompt", op="append", B=1, Q=49152, H=32, Hkv=8, D=128, tokens=1003, P=64, dtype="fp16",
             ragged=False, layers=1),
        # a step's bookkeeping, two forks of a session that write to the page they share, and what is thrown away
        dict(name="pages_step", op="pages", kind="step", streams=256, forks=32, tokens=3500, P=16, layers=2, Hkv=8,
             D=128, Q=17),
        # a pool after many sessions came and went, closed up
        dict(name="pages_compact", op="pages", kind="compact", streams=96, forks=0, tokens=4000, P=16, layers=4,
             Hkv=8, D=128, Q=1),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    dtype = rng.choice(("bf16", "fp16"))
    P = rng.choice((16, 16, 32, 64, 128))
    D = rng.choice((64, 128, 128))
    kind = rng.choice(("attend", "attend", "attend", "attend", "append", "step", "compact"))
    if kind == "attend":
        Hkv = rng.choice((1, 2, 4, 8, 16))
        g = rng.choice((1, 2, 3, 4, 5, 7, 8))
        Q = rng.choice((1, 1, log_int(2, 33), 17, log_int(34, 1500)))
        B = log_int(1, 128) if Q <= 33 else log_int(1, 4)
        # neither the cache nor the products go beyond the largest listed case
        room = min(64 * 12000 * 8 * 128 // (B * Hkv * D), 2048 * 20011 * 28 * 128 // (B * Hkv * g * D * Q))
        tokens = log_int(1, max(2, min(250000, room)))
        window = rng.choice((0, 0, 0, log_int(1, 2 * tokens)))
        return dict(op="attend", B=B, Q=Q, H=Hkv * g, Hkv=Hkv, D=D, tokens=tokens, P=P, dtype=dtype,
                    ragged=rng.random() < 0.7, window=window, layers=rng.choice((1, 2)))
    if kind == "append":
        Hkv = rng.choice((1, 2, 4, 8, 16))
        Q = rng.choice((1, 17, log_int(2, 33), log_int(34, 40000)))
        B = log_int(1, max(1, min(512, 49152 * 8 * 128 // (Q * Hkv * D))))
        return dict(op="append", B=B, Q=Q, H=Hkv * rng.choice((1, 4, 7)), Hkv=Hkv, D=D, tokens=log_int(1, 2000), P=P,
                    dtype=dtype, ragged=rng.random() < 0.7, layers=rng.choice((1, 2)))
    streams = log_int(2, 512) if kind == "step" else log_int(2, 128)
    page = 18 * D * (P // 16)
    layers = log_int(1, 4)
    Hkv = rng.choice((1, 2, 4, 8))
    tokens = log_int(20, max(21, min(8000, 96 * 4000 * 32 * 144 * 16 // (streams * layers * Hkv * page))))
    return dict(op="pages", kind=kind, streams=streams, forks=rng.randrange(0, streams // 2) if kind == "step" else 0,
                tokens=tokens, P=P, layers=layers, Hkv=Hkv, D=D, Q=rng.choice((1, 4, 9, 17, 33)))


def _lengths(case):
    """Context lengths of the streams before this pass; the same set for every seed."""
    n = case.get("B") or case["streams"]
    t = case["tokens"]
    if not case.get("ragged", True):
        return [max(0, t - i) for i in range(n)]
    return [int(t * (0.1 + 0.9 * (0.6180339887498949 * i % 1.0))) if i else t for i in range(n)]


def _counts(case):
    """New tokens of the streams: full proposals and shorter ones."""
    n, Q = case.get("B") or case["streams"], case["Q"]
    if not case.get("ragged", True):
        return [Q] * n
    return [Q - (i * 5) % ((Q + 1) // 2 + 1) if i else Q for i in range(n)]


# ------------------------------------------------------------------------------------------------ the format, plainly
def _quantise(x, exp):
    """float32 [..., D] -> (codes uint8 [..., D], scale bytes uint8 [..., D/16])."""
    b = x.float().unflatten(-1, (-1, 16)) * 2.0 ** -exp
    amax = b.abs().amax(-1)
    nan = b.isnan().any(-1)
    s = (amax / 6).clamp(max=448.0).nan_to_num(nan=0.0).to(torch.float8_e4m3fn)
    y = (b.abs() / s.float()[..., None])
    code = torch.zeros_like(y, dtype=torch.uint8)
    for t, even in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)):
        code += (y >= t) if even else (y > t)
    code += (b.signbit()).to(torch.uint8) * 8
    code *= ((s.float() > 0) & ~nan)[..., None]
    scale = s.view(torch.uint8) * ~nan + nan * torch.tensor(0x7F, dtype=torch.uint8, device=x.device)
    return code.flatten(-2), scale


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


# ------------------------------------------------------------------------------------------------ states
def _pool(case, n_pages, gen):
    """Pages of normally distributed keys (channels of unequal size) and values."""
    L, Hkv, P, D = case["layers"], case["Hkv"], case["P"], case["D"]
    pages = torch.empty(n_pages, L, Hkv, P // 16, 18 * D, dtype=torch.uint8, device=DEV)
    if case["op"] == "pages":                 # pages are moved, not read
        pages.view(torch.int32).random_(generator=gen)
        return pages
    size = torch.exp(0.4 * torch.randn(L, Hkv, 1, 1, D, generator=gen, device=DEV))
    step = max(1, (1 << 26) // (L * Hkv * P * D))
    for at in range(0, n_pages, step):
        kc, vc, ks, vs = _split(pages[at:at + step], D)
        shape = kc.shape[:-1] + (D,)
        for c, s, exp, mul in ((kc, ks, K_EXP, size), (vc, vs, V_EXP, 0.5)):
            code, scale = _quantise(torch.randn(shape, generator=gen, device=DEV) * mul, exp)
            c.copy_(_nibbles(code))
            s.copy_(scale)
    return pages


def _handle(state, case):
    """What a program that uses the package keeps: the cache object over the tensors, and its workspace."""
    import paper_2512_18337_b200 as S
    b = state["book"]
    state["cache"] = S.SamCache(n_pages=b["ref_count"].numel(), page_tokens=case["P"], n_streams=b["seq_len"].numel(),
                                max_pages=b["page_table"].shape[1], n_layers=case["layers"], n_kv_heads=case["Hkv"],
                                head_dim=case["D"], k_exp=K_EXP, v_exp=V_EXP, device=DEV,
                                tensors=dict(pages=state["pages"], **b))


def _book(n_streams, max_pages, n_pages):
    """The bookkeeping of a cache, in one tensor (so that it can be put back in one copy) and as its parts."""
    sizes = [n_streams * max_pages, n_streams, n_pages, n_pages, 4]
    flat = torch.zeros(sum(sizes), dtype=torch.int32, device=DEV)
    t, l, r, f, m = flat.split(sizes)
    return flat, dict(page_table=t.view(n_streams, max_pages), seq_len=l, ref_count=r, free_list=f, meta=m)


def _fill(book, lengths, P, extra, gen):
    """Tables over pages in no order, `extra` more tokens of each stream reserved; what is left is free."""
    n_streams, max_pages = book["page_table"].shape
    n_pages = book["ref_count"].numel()
    order = torch.randperm(n_pages, generator=gen, device=DEV).int()
    held = -(-(lengths + extra) // P)
    first = torch.cumsum(held, 0) - held
    at = torch.arange(max_pages, device=DEV)[None]
    has = at < held[:, None]
    book["page_table"].copy_(torch.where(has, order[(first[:, None] + at).clamp(max=n_pages - 1)], -1))
    book["seq_len"].copy_(lengths)
    book["ref_count"].zero_()
    book["ref_count"][book["page_table"][has].long()] = 1
    used = int(held.sum())
    book["free_list"].zero_()
    book["free_list"][:n_pages - used] = order[used:]
    book["meta"].copy_(torch.tensor([n_pages - used, 0, 0, 0]))


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    P, D, Q = case["P"], case["D"], case["Q"]
    lengths, counts = _lengths(case), _counts(case)
    n = len(lengths)
    perm = torch.randperm(n, generator=gen, device=DEV)
    seq = torch.tensor(lengths, device=DEV)[perm]
    new = torch.tensor(counts, dtype=torch.int32, device=DEV)[torch.randperm(n, generator=gen, device=DEV)]
    state = dict(case=case, n_new=new)
    if case["op"] in ("attend", "append"):
        B, H, Hkv = case["B"], case["H"], case["Hkv"]
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float16
        max_pages = -(-(max(lengths) + Q) // P)
        n_pages = sum(-(-(l + Q) // P) for l in lengths) + 3
        state["flat"], state["book"] = _book(B, max_pages, n_pages)
        _fill(state["book"], seq, P, Q, gen)
        state["pages"] = _pool(case, n_pages, gen)
        # queries, keys and values are slices of the projection's output
        qkv = torch.randn(B, Q, H + 2 * Hkv, D, generator=gen, device=DEV)
        qkv[:, :, H + Hkv:] *= 0.5
        state["qkv"] = qkv.to(dt)
        state["layer"] = case["layers"] - 1
    else:
        forks = case["forks"]
        max_pages = -(-(max(lengths) + Q) // P)
        spare = case["streams"] * (-(-Q // P) + 1) + forks + 5
        total = sum(-(-l // P) for l in lengths) + spare
        n_pages = total if case["kind"] == "step" else total + total // 2
        # streams that nothing runs on yet take the forks
        state["flat"], state["book"] = _book(n + forks, max_pages, n_pages)
        zeros = torch.zeros(forks, dtype=seq.dtype, device=DEV)
        _fill(state["book"], torch.cat([seq, zeros]), P, 0, gen)
        state["first"] = state["flat"].clone()
        state["pages"] = _pool(case, n_pages, gen)
        some = torch.randperm(n, generator=gen, device=DEV)
        state["src"] = some[:forks].int()
        state["dst"] = torch.arange(n, n + forks, dtype=torch.int32, device=DEV)
        state["n_new"] = torch.cat([new, new[:forks]])
        keep = torch.rand(n + forks, generator=gen, device=DEV)
        state["n_keep"] = (1 + (keep * state["n_new"]).int()).clamp(max=Q).minimum(state["n_new"])
        gone = torch.zeros(n + forks, dtype=torch.int32, device=DEV)
        gone[some[forks // 2:forks]] = DROP
        gone[n:n + forks // 2] = DROP
        state["n_back"] = gone
    if own:
        _handle(state, case)
    return state


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if case["op"] == "attend":
        return _attend(state)
    if case["op"] == "append":
        return _append(state)
    return _pages(state)


def _attend(state):
    """Attention of the new rows; their keys and values are in the cache already."""
    case, H = state["case"], state["case"]["H"]
    q = state["qkv"][:, :, :H]
    scale = case["D"] ** -0.5
    if own:
        return state["cache"].attend(state["layer"], q, n_new=state["n_new"], scale=scale, window=case["window"])
    return _attend_plain(state, q, scale)


def _attend_plain(state, q, scale):
    case, book = state["case"], state["book"]
    B, Q, H, Hkv, D, P = (case[x] for x in ("B", "Q", "H", "Hkv", "D", "P"))
    g = H // Hkv
    table = book["page_table"]
    tiles = state["pages"][table.clamp(min=0).long(), state["layer"]]             # [B, M, Hkv, P/16, 18 D]
    kc, vc, ks, vs = _split(tiles.transpose(1, 2), D)
    k = _values(kc, ks, K_EXP).reshape(B, Hkv, -1, D)
    pos = torch.arange(k.shape[2], device=DEV)
    row = book["seq_len"][:, None] + torch.arange(Q, device=DEV)                  # [B, Q] position of each row
    seen = (pos <= row[..., None]) & (table >= 0).repeat_interleave(P, 1)[:, None]
    if case["window"]:
        seen &= pos > row[..., None] - case["window"]
    seen &= (torch.arange(Q, device=DEV) < state["n_new"][:, None])[..., None]
    x = q.float().view(B, Q, Hkv, g, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, Q * g, D)
    s = torch.matmul(x, k.transpose(-1, -2)).mul_(scale).view(B, Hkv, Q, g, -1)
    del k
    s.masked_fill_(~seen[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    s.sub_(m.nan_to_num(neginf=0.0)).exp_()
    l = s.sum(-1, keepdim=True)
    v = _values(vc, vs, V_EXP).reshape(B, Hkv, -1, D)
    o = torch.matmul(s.view(B, Hkv, Q * g, -1), v).view(B, Hkv, Q, g, D)
    o = torch.where(l > 0, o / l, 0.0).permute(0, 2, 1, 3, 4).reshape(B, Q, H, D)
    lse = (m + l.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, Q, H)
    return o.to(q.dtype), lse


def _append(state):
    """New keys and values into the cache, and back as the values that later steps will see."""
    case, book = state["case"], state["book"]
    H, Hkv, Q = case["H"], case["Hkv"], case["Q"]
    k, v = state["qkv"][:, :, H:H + Hkv], state["qkv"][:, :, H + Hkv:]
    if own:
        c = state["cache"]
        c.append(state["layer"], k, v, n_new=state["n_new"])
        return c.read(state["layer"], first=book["seq_len"], n=state["n_new"], max_n=Q, dtype=k.dtype)
    return _append_plain(state, k, v)


def _append_plain(state, k, v):
    case, book = state["case"], state["book"]
    Q, P, D = case["Q"], case["P"], case["D"]
    i = torch.arange(Q, device=DEV)
    pos = book["seq_len"][:, None] + i                                            # [B, Q]
    page = book["page_table"].gather(1, (pos // P).long())
    on = (i < state["n_new"][:, None]) & (page >= 0)
    kc, vc, ks, vs = _split(state["pages"][:, state["layer"]], D)                 # [pages, Hkv, P/16, 16, ...]
    at = (page[on].long(), slice(None), (pos[on] % P // 16).long(), (pos[on] % 16).long())
    out = []
    for x, codes, scales, exp in ((k, kc, ks, K_EXP), (v, vc, vs, V_EXP)):
        code, scale = _quantise(x[on], exp)
        codes[at] = _nibbles(code)
        scales[at] = scale
        y = torch.zeros_like(x, memory_format=torch.contiguous_format)
        y[on] = _values(codes[at], scales[at], exp).to(x.dtype)
        out.append(y)
    return tuple(out)


def _pages(state):
    """A step's page work, or a pool closed up.  The bookkeeping is put back first, so that every pass finds the same."""
    case, book = state["case"], state["book"]
    state["flat"].copy_(state["first"])
    if case["kind"] == "compact":
        state["cache"].compact() if own else _compact_plain(state)
    elif own:
        c = state["cache"]
        if case["forks"]:
            c.fork(state["src"], state["dst"])
        c.reserve(state["n_new"])
        c.commit(state["n_keep"])
        c.commit(state["n_back"])
    else:
        if case["forks"]:
            _fork_plain(state)
        _reserve_plain(state)
        _commit_plain(book, state["n_keep"], case["P"])
        _commit_plain(book, state["n_back"], case["P"])
    return dict(page_table=book["page_table"], seq_len=book["seq_len"], ref_count=book["ref_count"],
                free_list=book["free_list"], meta=book["meta"][:2], pages=state["pages"].view(torch.int32))


def _fork_plain(state):
    """Each destination gets the source's committed pages; they are held once more."""
    book, src, dst = state["book"], state["src"].long(), state["dst"].long()
    held = -(-book["seq_len"][src] // state["case"]["P"])
    rows = book["page_table"][src]
    on = (torch.arange(rows.shape[1], device=DEV) < held[:, None]) & (rows >= 0)
    book["page_table"][dst] = torch.where(on, rows, -1)
    book["seq_len"][dst] = book["seq_len"][src]
    book["ref_count"] += torch.bincount(rows[on], minlength=book["ref_count"].numel()).int()


def _reserve_plain(state):
    """Pages for the new tokens, and copies of the shared pages that they will be written to."""
    case, book = state["case"], state["book"]
    P = case["P"]
    table, ref, free, meta = (book[x] for x in ("page_table", "ref_count", "free_list", "meta"))
    n = state["n_new"].clamp(min=0)
    rows = torch.arange(n.numel(), device=DEV)
    first = book["seq_len"] // P
    at = first[:, None] + torch.arange(-(-case["Q"] // P) + 1, device=DEV)
    on = (at < -(-(book["seq_len"] + n) // P)[:, None]) & (n > 0)[:, None]
    page = torch.where(on, table.gather(1, at.clamp(max=table.shape[1] - 1).long()), -2)
    # the last row that writes to a shared page keeps it, if all its holders write
    writes = (page[:, 0] >= 0) & (book["seq_len"] % P != 0)
    held = torch.where(writes, page[:, 0], 0).long()
    writers = torch.zeros_like(ref).index_add_(0, held, writes.int())
    last = torch.full_like(ref, -1, dtype=torch.int64).scatter_reduce_(0, held, torch.where(writes, rows, -1), "amax")
    copies = writes & ~((writers[held] == ref[held]) & (last[held] == rows))
    need = page == -1
    need[:, 0] |= copies
    flat = need.flatten()
    nth = torch.cumsum(flat, 0) - 1
    got = free[(meta[0] - 1 - nth).clamp(min=0)][flat]
    old, new = page[:, 0][copies].long(), torch.zeros_like(flat, dtype=torch.int32)
    new[flat] = got
    new = new.view(page.shape)
    state["pages"][new[:, 0][copies].long()] = state["pages"][old]
    ref -= torch.bincount(old, minlength=ref.numel()).int()
    ref[got.long()] = 1
    r, c = need.nonzero(as_tuple=True)
    table[r, at[r, c].long()] = new[r, c]
    meta[0] -= flat.sum()


def _commit_plain(book, n_keep, P):
    """Lengths move on (or back); pages beyond them lose a holder, and go onto the free list in order of rows."""
    table, ref, free, meta = (book[x] for x in ("page_table", "ref_count", "free_list", "meta"))
    new = (book["seq_len"].long() + n_keep).clamp(0, table.shape[1] * P)
    book["seq_len"].copy_(new)
    at = torch.arange(table.shape[1], device=DEV)
    beyond = (at >= -(-new // P)[:, None]) & (table >= 0)
    gone = table[beyond].long()
    table.masked_fill_(beyond, -1)
    ref -= torch.bincount(gone, minlength=ref.numel()).int()
    first = torch.full((ref.numel(),), gone.numel(), device=DEV)
    first.scatter_reduce_(0, gone, torch.arange(gone.numel(), device=DEV), "amin")
    freed = gone[(ref[gone] == 0) & (first[gone] == torch.arange(gone.numel(), device=DEV))].int()
    free[meta[0] + torch.arange(freed.numel(), device=DEV)] = freed
    meta[0] += freed.numel()


def _compact_plain(state):
    """Live pages beyond the number of live pages move to the free ids below it; the free list is in order."""
    book = state["book"]
    ref, table = book["ref_count"], book["page_table"]
    n = ref.numel()
    live = ref > 0
    total = live.sum()
    ids = torch.arange(n, device=DEV)
    src = (live & (ids >= total)).nonzero().squeeze(1)
    dst = (~live & (ids < total)).nonzero().squeeze(1)
    state["pages"][dst] = state["pages"][src]
    new = ids.int()
    new[src] = dst.int()
    ref[dst] = ref[src]
    ref[src] = 0
    table.copy_(torch.where(table >= 0, new[table.clamp(min=0).long()], -1))
    n_free = n - total
    book["free_list"].copy_(torch.where(ids < n_free, n - 1 - ids, book["free_list"]))
    book["meta"][0] = n_free


# ------------------------------------------------------------------------------------------------ in 64 bits
def _round_e2m1(y):
    """Nearest e2m1 value of a magnitude, ties to the even code."""
    q = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0)).double()
    return (torch.round(y / q) * q).clamp(max=6.0)


def _round_e4m3(v):
    q = torch.exp2(torch.floor(torch.log2(v.clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / q) * q).clamp(max=448.0)


def _read_exact(book, pages, layer, row, head, D, P, which):
    """All tokens [T, D] of one row and head of the cache in 64 bits, from the bit fields."""
    t = book["page_table"][row]
    tile = pages[t.clamp(min=0).long(), layer, head].reshape(-1, 18 * D)
    codes = tile[:, which * 8 * D:(which + 1) * 8 * D].reshape(-1, D // 2)
    scales = tile[:, (16 + which) * D:(17 + which) * D].reshape(-1, D // 16).double()
    nib = torch.stack([codes & 15, codes >> 4], -1).reshape(-1, D).double()
    sign = 1 - 2 * torch.floor(nib / 8)
    e, f = torch.floor(nib % 8 / 2), nib % 2
    mag = torch.where(e > 0, (2 + f) * torch.exp2(e - 2), f / 2)
    se, sf = torch.floor(scales / 8), scales % 8
    s = torch.where(se > 0, (8 + sf) * torch.exp2(se - 10), sf * 2.0 ** -9)
    return sign * mag * s.repeat_interleave(16, -1) * 2.0 ** (V_EXP if which else K_EXP)


def exact(case, seed):
    if case["op"] == "pages":
        return None
    state = prepare(case, seed)
    book, pages, layer = state["book"], state["pages"], state["layer"]
    B, Q, H, Hkv, D, P = (case[x] for x in ("B", "Q", "H", "Hkv", "D", "P"))
    n_new, seq = state["n_new"].tolist(), book["seq_len"].tolist()
    qkv = state["qkv"]
    if case["op"] == "append":
        out = []
        for at, exp in ((H, K_EXP), (H + Hkv, V_EXP)):
            x = qkv[:, :, at:at + Hkv].double().unflatten(-1, (-1, 16))
            s = _round_e4m3(x.abs().amax(-1, keepdim=True) / (6 * 2.0 ** exp)) * 2.0 ** exp
            y = torch.where(s > 0, x.sign() * _round_e2m1(x.abs() / s) * s, 0.0).flatten(-2)
            for b in range(B):
                y[b, n_new[b]:] = 0
            out.append(y)
        return tuple(out)
    g = H // Hkv
    out = torch.zeros(B, Q, H, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, Q, H), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(B):
        n, end = n_new[b], seq[b] + n_new[b]
        if n < 1:
            continue
        row = seq[b] + torch.arange(n, device=DEV)[:, None]
        pos = torch.arange(end, device=DEV)
        hidden = pos > row
        if case["window"]:
            hidden |= pos <= row - case["window"]
        for h in range(Hkv):
            k = _read_exact(book, pages, layer, b, h, D, P, 0)[:end]
            v = _read_exact(book, pages, layer, b, h, D, P, 1)[:end]
            x = qkv[b, :n, h * g:(h + 1) * g].double()
            s = (torch.einsum("ngd,td->gnt", x, k) / math.sqrt(D)).masked_fill(hidden, -math.inf)
            lse[b, :n, h * g:(h + 1) * g] = torch.logsumexp(s, -1).T
            out[b, :n, h * g:(h + 1) * g] = (torch.softmax(s, -1) @ v).transpose(0, 1)
    return out, lse


# ------------------------------------------------------------------------------------------------ what a pass needs
def work(case):
    P, D, Hkv = case["P"], case["D"], case["Hkv"]
    lengths, counts = _lengths(case), _counts(case)
    if case["op"] == "attend":
        H, w = case["H"], case["window"]
        mean = sum(counts) / len(counts)
        kv = pairs = 0.0
        for l in lengths:                       # lengths and counts meet in another order for each seed
            first = max(0, l - w + 1) if w else 0
            kv += l + mean - first
            full = mean * l + mean * (mean + 1) / 2
            pairs += min(full, mean * w) if w else full
        rows = sum(counts) * H
        out = len(lengths) * case["Q"] * H
        return {"bytes": kv * Hkv * D * 9 / 8 + rows * D * 2 + out * (D * 2 + 4), "flops": 4 * D * H * pairs}
    if case["op"] == "append":
        n, every = sum(counts) * Hkv * D * 2, len(counts) * case["Q"] * Hkv * D * 2
        # keys and values in 16 bits, into the cache, out of it, and in 16 bits again
        return {"bytes": n * 2 + 2 * n * 9 / 16 + every * 2, "flops": 0}
    page = case["layers"] * Hkv * (P // 16) * 18 * D
    held = sum(-(-l // P) for l in lengths)
    if case["kind"] == "compact":
        spare = case["streams"] * (-(-case["Q"] // P) + 1) + 5
        n_pages = held + spare + (held + spare) // 2
        return {"bytes": 2 * page * held * (1 - held / n_pages) + 8 * n_pages + 8 * held, "flops": 0}
    shared = case["forks"] * held / case["streams"]
    # a fork and its source both write to the page that they share: one of the two gets a copy
    copies = case["forks"] * (1 - 1 / P)
    return {"bytes": 2 * page * copies + 8 * (shared + case["forks"]) + 4 * 4 * (case["streams"] + case["forks"]), "flops": 0}
