"""What the paged 4-bit key/value cache is measured on: its plan (block tables and slot maps from request lengths), the
cache itself (append and read back) and the attention that reads it, with a plain form of each in elementary torch
operations.

The cache's memory format is written out here once more (``_FORMAT`` below), because the plain forms work on the same
bytes as the kernels do.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

# _FORMAT.  pages: uint8 [n_pages, kv_heads, page / 16, tile bytes].  A tile holds 16 tokens of one head: for every group
# of 64 head dimensions 512 bytes of key codes, then the same for the values, then the parameters.  Codes come in 32-bit
# words of 8 consecutive dimensions e8 = (dim % 64) / 8; the code of dimension j of the 8 sits at bits
# 4 (j / 2) + 16 (j % 2).  Word of token t (0..15) inside a group:
#   keys:    16 (t % 8) + 4 (e8 / 2) + 2 (t / 8) + e8 % 2
#   values:  16 e8 + 4 (t % 8 / 2) + 2 (t / 8) + t % 2
# Parameters: per token the (scale, zero) pairs in fp16, one per key group, then one per value group.
# The value of a code is scale * code + zero.  Of a group x: zero = fp16(min), scale = fp16((max - min) * fp32(1 / 15)),
# code = round((x - zero) * (1 / scale)) within 0..15, every step rounded to fp32; NaN counts as 0, and what lies beyond
# +-65504 as +-65504.
GROUP = 64
TILE = 16
_SHIFT = (0, 16, 4, 20, 8, 24, 12, 28)


def _tile_bytes(dim):
    return (dim // GROUP) * (2 * 512 + TILE * 8)


# ------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # a decode step's bookkeeping for a handful of requests: pure latency
        dict(name="plan_decode", op="plan", requests=8, page=16, min_ctx=100, max_ctx=1200, min_new=1, max_new=1, finished=0),
        # a large server's step: prompts, chunks and single tokens together, finished requests giving their pages back
        dict(name="plan_mixed", op="plan", requests=2048, page=64, min_ctx=0, max_ctx=8000, min_new=1, max_new=256, finished=16),
        # one decoder layer's prompt (1024 tokens, 32 heads) written to the cache, k and v being slices of a fused projection
        dict(name="cache_prompt", op="cache", requests=1, tokens=1024, kv_heads=32, dim=128, page=64, dtype="bf16", fused=True),
        # the new tokens of a small decode batch, a narrow model in fp32: latency
        dict(name="cache_decode", op="cache", requests=13, tokens=13, kv_heads=8, dim=64, page=16, dtype="f32", fused=False),
        # many prompts at once with grouped heads
        dict(name="cache_bulk", op="cache", requests=24, tokens=16384, kv_heads=8, dim=128, page=64, dtype="bf16", fused=True),
        # the decoder's own decode step: one token, 32 heads, a prompt of 1024 and 128 generated tokens in the cache
        dict(name="decode_single", op="attend", requests=1, heads=32, kv_heads=32, dim=128, page=64, dtype="bf16",
             min_ctx=1151, max_ctx=1151, min_new=1, max_new=1, causal=True, window=0),
        # a serving batch of grouped-head decode steps with ragged lengths
        dict(name="decode_batch", op="attend", requests=64, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16",
             min_ctx=500, max_ctx=8000, min_new=1, max_new=1, causal=True, window=0),
        # one long document
        dict(name="decode_long", op="attend", requests=1, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16",
             min_ctx=131070, max_ctx=131070, min_new=1, max_new=1, causal=True, window=0),
        # a small fp32 model, three query heads to a kv head, several drafted tokens per request, some requests empty
        dict(name="decode_f32", op="attend", requests=9, heads=6, kv_heads=2, dim=64, page=16, dtype="f32",
             min_ctx=0, max_ctx=2000, min_new=0, max_new=4, causal=True, window=0),
        # the decoder's prompt: 1024 tokens, 32 heads, causal
        dict(name="prompt_single", op="attend", requests=1, heads=32, kv_heads=32, dim=128, page=64, dtype="bf16",
             min_ctx=0, max_ctx=0, min_new=1024, max_new=1024, causal=True, window=0),
        # prompts in chunks behind cached context, grouped heads, ragged
        dict(name="prompt_chunks", op="attend", requests=6, heads=32, kv_heads=8, dim=128, page=64, dtype="bf16",
             min_ctx=100, max_ctx=4100, min_new=65, max_new=2049, causal=True, window=0),
        # fp32 prompts with a sliding window
        dict(name="prompt_f32", op="attend", requests=3, heads=12, kv_heads=4, dim=64, page=32, dtype="f32",
             min_ctx=0, max_ctx=300, min_new=33, max_new=517, causal=True, window=256),
    ]


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = max(lo, min(hi, n))
    return n + 1 if n == 3072 else n


def draw(rng):
    """One more case: a plan, a cache or an attention call of the listed ones' ranges."""
    kind = rng.choice(("plan", "cache", "decode", "decode", "prompt", "prompt"))
    page = rng.choice((16, 32, 64, 128))
    if kind == "plan":
        most = rng.choice((1, 1, _log_int(rng, 2, 256)))
        return dict(op="plan", requests=_log_int(rng, 1, 2048), page=page, min_ctx=0, max_ctx=_log_int(rng, 16, 8000),
                    min_new=rng.choice((0, 1)), max_new=most, finished=rng.choice((0, 0, 3, 16)))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    dim = rng.choice((64, 128, 128))
    kv_heads = rng.choice((1, 2, 4, 8, 8, 32))
    if kind == "cache":
        requests = _log_int(rng, 1, 64)
        most = 16384 * 8 * 128 // (kv_heads * dim) // (2 if dtype == "f32" else 1)
        return dict(op="cache", requests=requests, tokens=max(requests, _log_int(rng, 1, min(most, 32768))), kv_heads=kv_heads,
                    dim=dim, page=page, dtype=dtype, fused=rng.choice((True, False)))
    ratio = rng.choice((1, 2, 3, 4, 4, 5, 8) if kv_heads <= 8 else (1, 2))
    window = rng.choice((0, 0, 0, _log_int(rng, 17, 2000)))
    if kind == "decode":
        requests = _log_int(rng, 1, 128)
        longest = max(1, min(131070, 180000 * 8 // (kv_heads * requests)))
        hi = _log_int(rng, 1, longest)
        return dict(op="attend", requests=requests, heads=kv_heads * ratio, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype,
                    min_ctx=rng.choice((0, hi // 8, hi)), max_ctx=hi, min_new=rng.choice((0, 1, 1)), max_new=rng.choice((1, 1, 1, 2, 5)),
                    causal=rng.choice((True, True, False)), window=window)
    requests = _log_int(rng, 1, 6)
    heads = kv_heads * ratio
    hi_new = _log_int(rng, 33, max(64, min(2049, 2049 * 32 * 6 // (heads * requests) // (4 if dtype == "f32" else 1))))
    hi_ctx = rng.choice((0, _log_int(rng, 10, 4100)))
    return dict(op="attend", requests=requests, heads=heads, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype,
                min_ctx=rng.choice((0, hi_ctx // 2)), max_ctx=hi_ctx, min_new=rng.choice((1, hi_new // 3 + 1, hi_new)), max_new=hi_new,
                causal=rng.choice((True, True, True, False)), window=window)


def _spread(n, lo, hi, phase):
    """n whole numbers from lo to hi, spread over their logarithm (golden-ratio sequence; the ends among them)."""
    if n == 1:
        return [hi]
    out = []
    for i in range(n):
        u = 0.0 if i == 0 else 1.0 if i == 1 else (phase + 0.6180339887498949 * i) % 1.0
        v = max(lo, min(hi, int(round(math.exp(math.log(lo + 1) + u * (math.log(hi + 1) - math.log(lo + 1)))) - 1)))
        out.append(v + 1 if v == 3072 else v)
    return out


def _lengths(case):
    """(context, new) lengths of the case's requests: the same for every seed, which only deals them out differently.
    A request whose new length is -1 has finished (plans only)."""
    n = case["requests"]
    ctx = _spread(n, case["min_ctx"], case["max_ctx"], 0.1)
    new = _spread(n, case["min_new"], case["max_new"], 0.4)
    new = new[n // 2:] + new[:n // 2]          # the longest chunk does not always meet the longest context
    if case.get("finished"):
        new = [-1 if i % case["finished"] == 2 else v for i, v in enumerate(new)]
    return ctx, new


def _dealt(case, seed):
    ctx, new = _lengths(case)
    order = np.random.RandomState((seed * 7919 + 13) % (1 << 31)).permutation(len(ctx))
    return np.array(ctx, dtype=np.int64)[order], np.array(new, dtype=np.int64)[order]


def _cache_lengths(case):
    """Tokens of each request of a cache case: near-equal ragged shares of `tokens`, and where in the request they start."""
    n, t = case["requests"], case["tokens"]
    cut = [0]
    for i in range(1, n):
        cut.append(min(t - (n - i), max(cut[-1] + 1, round(t * i / n) + (7 * i) % 5 - 2)))
    cut.append(t)
    new = [b - a for a, b in zip(cut, cut[1:])]
    ctx = [(37 * i) % 150 if n > 1 else 0 for i in range(n)]
    return ctx, new


# ----------------------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed % (1 << 62))
    return g


def _ints(v, dtype=torch.int32):
    return torch.tensor(np.asarray(v), dtype=dtype, device=DEV)


def _tables(ctx, new, page, seed, spare=0):
    """Block table over randomly placed pages for requests that hold ctx + new tokens, and the number of pages."""
    blocks = [-(-int(a + b) // page) for a, b in zip(ctx, new)]
    most = max(1, max(blocks))
    total = sum(blocks) + spare
    pages = np.random.RandomState((seed * 31 + 5) % (1 << 31)).permutation(max(1, total))
    table = np.full((len(blocks), most), -1, dtype=np.int32)
    at = 0
    for r, n in enumerate(blocks):
        table[r, :n] = pages[at:at + n]
        at += n
    return table, max(1, total)


def _slots(ctx, new, table, page):
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, new)] or [np.zeros(0, dtype=np.int64)]).astype(np.int64)
    req = np.repeat(np.arange(len(ctx)), new)
    return table[req, pos // page].astype(np.int64) * page + pos % page


def _keys_values(tokens, heads, dim, g):
    """Keys with a few channels far from zero, as rotary models have them, and plain values: fp32 [tokens, heads, dim]."""
    k = torch.randn(tokens, heads, dim, generator=g, device=DEV)
    off = torch.randn(heads, dim, generator=g, device=DEV) * 3 * (torch.rand(heads, dim, generator=g, device=DEV) < 0.05)
    v = torch.randn(tokens, heads, dim, generator=g, device=DEV)
    return k.add_(off), v


def _attend_inputs(case, seed):
    """Lengths, q and the keys and values behind the cache, in the case's type."""
    ctx, new = _dealt(case, seed)
    g = _generator(seed)
    dt = DTYPES[case["dtype"]]
    k, v = _keys_values(int((ctx + new).sum()), case["kv_heads"], case["dim"], g)
    q = torch.randn(int(new.sum()), case["heads"], case["dim"], generator=g, device=DEV) * 1.5
    return ctx, new, q.to(dt), k.to(dt), v.to(dt)


def prepare(case, seed):
    page = case["page"]
    if case["op"] == "plan":
        ctx, new = _dealt(case, seed)
        live = np.maximum(new, 0)
        need = int(sum(-(-(c + n) // page) for c, n in zip(ctx, live)))
        most = max(1, int(max(-(-(c + n) // page) for c, n in zip(ctx, live))))
        n_pages = need + 7
        perm = np.random.RandomState((seed * 101 + 3) % (1 << 31)).permutation(n_pages).astype(np.int32)
        wide = np.full((len(ctx), most), -1, dtype=np.int32)
        used = 0
        for r, c in enumerate(ctx):
            n = -(-int(c) // page)
            wide[r, :n] = perm[used:used + n]
            used += n
        head = int(seed) % n_pages
        ring = np.full(n_pages, -1, dtype=np.int32)
        ring[(head + np.arange(n_pages - used)) % n_pages] = perm[used:]
        return dict(case=case, ctx_lens=_ints(ctx), new_lens=_ints(new), table=_ints(wide), ring=_ints(ring),
                    state=_ints([head, n_pages - used]), tokens=int(live.sum()))
    if case["op"] == "cache":
        ctx, new = _cache_lengths(case)
        table, n_pages = _tables(ctx, new, page, seed, spare=3)
        slots = _slots(ctx, new, table, page)
        g = _generator(seed)
        T, H, D, dt = case["tokens"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
        k, v = _keys_values(T, H, D, g)
        if case["fused"]:                        # [q | k | v] rows of one projection, a quarter as wide again for q
            rows = torch.zeros(T, 3, H, D, device=DEV, dtype=dt)
            rows[:, 1], rows[:, 2] = k.to(dt), v.to(dt)
            k, v = rows[:, 1], rows[:, 2]
        else:
            k, v = k.to(dt), v.to(dt)
        pages = torch.full((n_pages, H, page // TILE, _tile_bytes(D)), 255, dtype=torch.uint8, device=DEV)
        return dict(case=case, pages=pages, k=k, v=v, slots=torch.from_numpy(slots).to(DEV))
    ctx, new, q, k, v = _attend_inputs(case, seed)
    table, n_pages = _tables(ctx, new, page, seed, spare=2)
    pages = torch.full((n_pages, case["kv_heads"], page // TILE, _tile_bytes(case["dim"])), 255, dtype=torch.uint8, device=DEV)
    slots = torch.from_numpy(_slots(np.zeros_like(ctx), ctx + new, table, page)).to(DEV)
    _write(pages, k, v, slots)
    indptr = np.concatenate([[0], np.cumsum(new)])
    return dict(case=case, pages=pages, q=q, table=_ints(table), indptr=_ints(indptr), kv_lens=_ints(ctx + new),
                most_new=max(1, int(new.max())))


# ------------------------------------------------------------------------------------------------------- plain forms

def _quantise(x):
    """fp32 [..., dim] -> codes int32 [..., groups, 64] and (scale, zero) fp16 [..., groups, 2]."""
    x = torch.nan_to_num(x.unflatten(-1, (-1, GROUP)), nan=0.0, posinf=65504.0, neginf=-65504.0).clamp(-65504.0, 65504.0)
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s, z = ((hi - lo) * (1.0 / 15.0)).half(), lo.half()      # the constant is rounded to fp32
    inv = torch.where(s > 0, 1.0 / s.float(), torch.zeros_like(lo))
    c = torch.round((x - z.float()) * inv).clamp(0.0, 15.0).to(torch.int32)
    return c, torch.cat([s, z], -1)


def _words(c):
    """codes int32 [..., groups, 64] -> words int32 [..., groups, 8]."""
    shift = torch.tensor(_SHIFT, device=c.device, dtype=torch.int32)
    return (c.unflatten(-1, (8, 8)).to(torch.int32) << shift).sum(-1, dtype=torch.int32)


def _word_places(pages, slots):
    """Where a token's words sit, in int32 words of the pages: keys [T, H, G, 8], values alike, parameters [T, H, 2 G]."""
    _, H, tiles, nbytes = pages.shape
    G = nbytes // _tile_bytes(GROUP)
    page, at = slots // (tiles * TILE), slots % (tiles * TILE)
    t = at % TILE
    h = torch.arange(H, device=slots.device)
    base = (((page[:, None] * H + h) * tiles + (at // TILE)[:, None]) * (nbytes // 4))[:, :, None, None]
    e8 = torch.arange(8, device=slots.device)
    g = torch.arange(G, device=slots.device)[:, None] * 128
    t4 = t[:, None, None, None]
    kw = base + g + 16 * (t4 % 8) + 4 * (e8 // 2) + 2 * (t4 // 8) + e8 % 2
    vw = base + G * 128 + g + 16 * e8 + 4 * (t4 % 8 // 2) + 2 * (t4 // 8) + t4 % 2
    pw = base[..., 0] + 2 * G * 128 + t[:, None, None] * (2 * G) + torch.arange(2 * G, device=slots.device)
    return kw, vw, pw


def _write(pages, k, v, slots):
    kw, vw, pw = _word_places(pages, slots)
    kc, kp = _quantise(k.float())
    vc, vp = _quantise(v.float())
    flat = pages.view(torch.int32).view(-1)
    flat[kw.reshape(-1)] = _words(kc).reshape(-1)
    flat[vw.reshape(-1)] = _words(vc).reshape(-1)
    flat[pw.reshape(-1)] = torch.cat([kp, vp], 2).contiguous().view(torch.int32).reshape(-1)


def _values(words, params):
    """words int32 [..., G, 8], params fp16 [..., G, 2] -> fp32 [..., 64 G]."""
    shift = torch.tensor(_SHIFT, device=words.device, dtype=torch.int32)
    c = ((words[..., None] >> shift) & 15).flatten(-2).float()
    p = params.float()
    return (c * p[..., :1] + p[..., 1:]).flatten(-2)


def _read(pages, slots):
    kw, vw, pw = _word_places(pages, slots)
    flat = pages.view(torch.int32).view(-1)
    par = flat[pw].view(torch.float16).unflatten(-1, (2, -1, 2))
    return _values(flat[kw], par[:, :, 0]), _values(flat[vw], par[:, :, 1])


def _plain_plan(st):
    case, ctx, new, table = st["case"], st["ctx_lens"].long(), st["new_lens"].long(), st["table"].clone()
    page, n_pages, T = case["page"], st["ring"].numel(), st["tokens"]
    ring, head, count = st["ring"].clone(), st["state"][0].long(), st["state"][1].long()
    live = new.clamp(min=0)
    kv = torch.where(new < 0, torch.zeros_like(ctx), ctx + live)
    zero = torch.zeros(1, dtype=torch.int64, device=ctx.device)
    indptr = torch.cat([zero, live.cumsum(0)])
    had = (ctx + page - 1) // page
    want = torch.where(new < 0, had, (ctx + live + page - 1) // page)
    cols = torch.arange(table.shape[1], device=ctx.device)
    fresh = (cols >= had[:, None]) & (cols < want[:, None])          # cells that get a page
    nth = fresh.view(-1).cumsum(0).view(fresh.shape) - 1
    taken = fresh.sum()
    table = torch.where(fresh, ring[(head + nth.clamp(min=0)) % n_pages], table)
    gone = (new < 0)[:, None] & (cols < had[:, None])                # cells that give theirs back
    back = gone.view(-1).cumsum(0).view(gone.shape) - 1
    end = torch.full_like(back, n_pages)
    longer = torch.cat([ring, ring[:1]])
    longer[torch.where(gone, (head + count + back) % n_pages, end).view(-1)] = table.view(-1)
    ring = longer[:n_pages]
    token = torch.arange(T, device=ctx.device)
    req = torch.searchsorted(indptr, token, right=True) - 1
    pos = ctx[req] + token - indptr[req]
    slots = table[req, pos // page].long() * page + pos % page
    state = torch.stack([(head + taken) % n_pages, count - taken + gone.sum()])
    return dict(table=table, ring=ring, state=state.int(), indptr=indptr.int(), kv_lens=kv.int(), slots=slots, positions=pos.int())


def _plain_attend(st):
    case, pages, q, table = st["case"], st["pages"], st["q"], st["table"].long()
    H, Hk, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    R, nb = table.shape
    G, ratio = D // GROUP, H // Hk
    L, Q = nb * page, st["most_new"]
    indptr, kv = st["indptr"].long(), st["kv_lens"].long()
    new = indptr[1:] - indptr[:-1]
    # the cache as fp32 [R, Hk, L, D]
    tiles = pages.view(torch.int32)[table.clamp(min=0)].transpose(1, 2).reshape(R, Hk, L // TILE, -1)
    par = tiles[..., 2 * G * 128:].contiguous().view(torch.float16).view(R, Hk, L, 2, G, 2)
    kw = tiles[..., :G * 128].view(R, Hk, -1, G, 8, 4, 2, 2).permute(0, 1, 2, 6, 4, 3, 5, 7).reshape(R, Hk, L, G, 8)
    vw = tiles[..., G * 128:2 * G * 128].view(R, Hk, -1, G, 8, 4, 2, 2).permute(0, 1, 2, 6, 5, 7, 3, 4).reshape(R, Hk, L, G, 8)
    j = torch.arange(L, device=q.device)
    here = (j < kv[:, None])[:, None, :, None]
    k = torch.where(here, _values(kw, par[..., 0, :, :]), torch.zeros((), device=q.device))
    v = torch.where(here, _values(vw, par[..., 1, :, :]), torch.zeros((), device=q.device))
    # q padded to [R, Q, H, D], and the position of every row in its request
    i = torch.arange(Q, device=q.device)
    row = (indptr[:-1, None] + i).clamp(max=max(0, q.shape[0] - 1))
    pos = kv[:, None] - new[:, None] + i
    qs = q.float()[row].view(R, Q, Hk, ratio, D).permute(0, 2, 3, 1, 4).reshape(R, Hk, ratio * Q, D)
    s = (qs @ k.transpose(-1, -2)).view(R, Hk, ratio, Q, L) * (1.0 / math.sqrt(D))
    seen = (j < kv[:, None, None]) & (i < new[:, None])[..., None]
    if case["causal"]:
        seen = seen & (j <= pos[..., None])
    if case["window"]:
        seen = seen & (j > pos[..., None] - case["window"])
    s = s.masked_fill(~seen[:, None, None], float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    o = (p.view(R, Hk, ratio * Q, L) @ v).view(R, Hk, ratio, Q, D) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 3, 1, 2, 4).reshape(R * Q, H, D)
    token = torch.arange(q.shape[0], device=q.device)
    req = torch.searchsorted(indptr, token, right=True) - 1
    return o[req * Q + token - indptr[req]].to(q.dtype)


def run(st):
    op = st["case"]["op"]
    if own:
        from paper_2602_06822_b200 import pop
        if op == "plan":
            p = pop.kv_plan(st["ctx_lens"], st["new_lens"], st["table"], st["ring"], st["state"], st["case"]["page"], st["tokens"],
                            state_out=torch.empty_like(st["state"]))
            return dict(table=st["table"], ring=st["ring"], state=p.state, indptr=p.q_indptr, kv_lens=p.kv_lens, slots=p.slots,
                        positions=p.positions)
        if op == "cache":
            pop.kv_append(st["pages"], st["k"], st["v"], st["slots"])
            return pop.kv_read(st["pages"], st["slots"], st["k"].dtype)
        return pop.kv_attention(st["pages"], st["q"], st["table"], st["indptr"], st["kv_lens"], causal=st["case"]["causal"],
                                window=st["case"]["window"])
    if op == "plan":
        return _plain_plan(st)
    if op == "cache":
        _write(st["pages"], st["k"], st["v"], st["slots"])
        k, v = _read(st["pages"], st["slots"])
        return k.to(st["k"].dtype), v.to(st["v"].dtype)
    return _plain_attend(st)


# ------------------------------------------------------------------------------------------------------------ work

def _visible(ctx, new, causal, window):
    """(query, key) pairs that see each other, and the keys that any query of the request sees."""
    if new <= 0:
        return 0, 0
    n = ctx + new
    last = (lambda i: ctx + i + 1) if causal else (lambda i: n)
    first = (lambda i: max(0, ctx + i - window + 1)) if window else (lambda i: 0)
    return sum(last(i) - first(i) for i in range(new)), n - first(0)


def work(case):
    if case["op"] == "plan":
        ctx, new = _lengths(case)
        page, T = case["page"], sum(n for n in new if n > 0)
        pages = sum(-(-(c + n) // page) - -(-c // page) if n >= 0 else -(-c // page) for c, n in zip(ctx, new))
        return dict(bytes=8 * len(ctx) + 8 * pages + 8 * len(ctx) + 12 * T, flops=0)
    if case["op"] == "cache":
        T, H, D = case["tokens"], case["kv_heads"], case["dim"]
        e = 2 if case["dtype"] == "bf16" else 4
        return dict(bytes=4 * T * H * D * e + 2 * T * H * _tile_bytes(D) / TILE + 16 * T, flops=0)
    ctx, new = _lengths(case)
    H, Hk, D, e = case["heads"], case["kv_heads"], case["dim"], 2 if case["dtype"] == "bf16" else 4
    seen = [_visible(c, n, case["causal"], case["window"]) for c, n in zip(ctx, new)]
    keys, pairs = sum(s[1] for s in seen), sum(s[0] for s in seen)
    return dict(bytes=keys * Hk * _tile_bytes(D) / TILE + 2 * sum(new) * H * D * e + 4 * keys / case["page"] + 8 * len(ctx),
                flops=4.0 * pairs * H * D)


# ----------------------------------------------------------------------------------------------------------- exact

def _stored64(x):
    """What the cache holds for x [T, H, D], by the format's definition: scale and zero point rounded to binary16, the
    constant 1 / 15, the reciprocal, the differences and the products that decide them rounded to binary32, the value in
    64 bits."""
    T, H, D = x.shape
    out = torch.empty(T, H, D, dtype=torch.float64, device=x.device)
    for a in range(0, D, GROUP):
        y = x[:, :, a:a + GROUP].double()
        y = torch.where(y != y, torch.zeros_like(y), y).clamp(-65504.0, 65504.0)
        least, most = y.min(2, keepdim=True).values, y.max(2, keepdim=True).values
        scale = ((most - least).float().double() * float(np.float32(1.0 / 15.0))).float().half().double()
        zero = least.half().double()
        per = torch.where(scale == 0, torch.zeros_like(scale), (1.0 / scale).float().double())
        code = ((y - zero).float().double() * per).float().double().round().clamp(0, 15)
        out[:, :, a:a + GROUP] = zero + scale * code
    return out


def exact(case, seed):
    if case["op"] == "plan":
        return None
    if case["op"] == "cache":
        g = _generator(seed)
        k, v = _keys_values(case["tokens"], case["kv_heads"], case["dim"], g)
        dt = DTYPES[case["dtype"]]
        return _stored64(k.to(dt)), _stored64(v.to(dt))
    ctx, new, q, k, v = _attend_inputs(case, seed)
    if work(case)["flops"] > 1.5e12:
        return None
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    at_q = at_k = 0
    for c, n in zip(ctx.tolist(), new.tolist()):
        ks, vs = _stored64(k[at_k:at_k + c + n]), _stored64(v[at_k:at_k + c + n])
        for i0 in range(0, n, 256):
            i1 = min(n, i0 + 256)
            place = torch.arange(c + i0, c + i1, device=q.device)[:, None]
            key = torch.arange(c + n, device=q.device)[None, :]
            hide = torch.zeros(i1 - i0, c + n, dtype=torch.bool, device=q.device)
            if case["causal"]:
                hide |= key > place
            if case["window"]:
                hide |= key <= place - case["window"]
            for h in range(H):
                logits = q[at_q + i0:at_q + i1, h].double() @ ks[:, h // (H // Hk)].T / math.sqrt(D)
                logits[hide] = -math.inf
                peak = logits.max(1, keepdim=True).values
                weight = (logits - torch.where(peak == -math.inf, torch.zeros_like(peak), peak)).exp()
                norm = weight.sum(1, keepdim=True)
                out[at_q + i0:at_q + i1, h] = weight @ vs[:, h // (H // Hk)] / torch.where(norm == 0, torch.ones_like(norm), norm)
        at_q += n
        at_k += c + n
    return out
