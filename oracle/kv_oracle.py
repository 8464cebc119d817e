"""Plain numpy oracle of the paged 4-bit key / value cache (format and meaning as include/pop.h states them): loops and
64-bit sums, no code shared with the library."""
import numpy as np


def plan(ctx, new, table, ring, head, count, page, capacity):
    """One step's plan by walking over the requests; table and ring are copied.  Returns a dict of what pop_kv_plan writes."""
    table, ring = table.copy(), ring.copy()
    n_pages, max_blocks = len(ring), table.shape[1]
    indptr, kv_lens, slots, positions, given_back, want, got = [0], [], [], [], [], 0, 0
    for r, (c, n) in enumerate(zip(ctx, new)):
        had = -(-c // page)
        if n < 0:
            given_back += [int(p) for p in table[r, :min(had, max_blocks)] if 0 <= p < n_pages]
            kv_lens.append(0)
            indptr.append(indptr[-1])
            continue
        for b in range(had, -(-(c + n) // page)):
            want += 1
            if b < max_blocks:                       # the row has a place for it
                table[r, b] = -1
                if got < count:
                    table[r, b] = ring[(head + got) % n_pages]
                    got += 1
        for i in range(n):
            b = (c + i) // page
            p = int(table[r, b]) if b < max_blocks else -1
            slots.append(p * page + (c + i) % page if 0 <= p < n_pages else -1)
            positions.append(c + i)
        kv_lens.append(c + n)
        indptr.append(indptr[-1] + n)
    for i, p in enumerate(given_back):
        ring[(head + count + i) % n_pages] = p
    pad = max(0, capacity - len(slots))
    return dict(table=table, ring=ring, state=[(head + got) % n_pages, count - got + len(given_back)], q_indptr=indptr,
                kv_lens=kv_lens, slots=(slots + [-1] * pad)[:capacity], positions=(positions + [-1] * pad)[:capacity],
                info=[indptr[-1], want - got])


def quantise(x):
    """x float32 [..., 64] -> (codes, scale, zero), every step rounded to float32 / float16 as the format says."""
    x = np.where(np.isnan(x), np.float32(0), x).astype(np.float32)
    x = np.clip(x, np.float32(-65504), np.float32(65504))
    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    scale = ((hi - lo) * np.float32(1.0 / 15.0)).astype(np.float16)
    zero = lo.astype(np.float16)
    with np.errstate(divide="ignore"):
        inv = np.where(scale > 0, np.float32(1.0) / scale.astype(np.float32), np.float32(0))
    codes = np.clip(np.rint((x - zero.astype(np.float32)) * inv), 0, 15).astype(np.int64)
    return codes, scale[..., 0], zero[..., 0]


def stored(x):
    """The values (float64) that the cache holds for x float32 [tokens, heads, dim]."""
    y = x.reshape(x.shape[:-1] + (-1, 64))
    c, s, z = quantise(y)
    return (s.astype(np.float64)[..., None] * c + z.astype(np.float64)[..., None]).reshape(x.shape)


def tile_bytes(dim):
    return dim // 64 * (1024 + 128)


def unpack_token(pages, slot, head, dim):
    """(k, v) float64 [dim] of one slot, taken byte by byte from pages uint8 [n_pages, heads, tiles, bytes]."""
    page_size = pages.shape[2] * 16
    G = dim // 64
    tile = pages[slot // page_size, head, slot % page_size // 16]
    t = slot % 16
    words = tile.view(np.uint32)
    params = tile[G * 1024:].view(np.float16).reshape(16, 2, G, 2)
    out = np.zeros((2, dim))
    for d in range(dim):
        g, e8, j = d // 64, d % 64 // 8, d % 8
        at = (16 * (t % 8) + 4 * (e8 // 2) + 2 * (t // 8) + e8 % 2, 16 * e8 + 4 * (t % 8 // 2) + 2 * (t // 8) + t % 2)
        for kv in range(2):
            w = int(words[kv * G * 128 + g * 128 + at[kv]])
            c = w >> (4 * (j // 2) + 16 * (j % 2)) & 15
            out[kv, d] = float(params[t, kv, g, 0]) * c + float(params[t, kv, g, 1])
    return out


def attention(q, k, v, n_ctx, scale, causal, window, absent=None):
    """q [n, H, D], k and v [L, Hk, D] (float64; the request's keys, queries at positions n_ctx + i where n_ctx may be negative)
    -> out [n, H, D], lse [n, H].  absent: boolean [L], keys that are not there."""
    n, H, D = q.shape
    L, Hk = k.shape[:2]
    out, lse = np.zeros((n, H, D)), np.full((n, H), -np.inf)
    j = np.arange(L)
    for i in range(n):
        p = n_ctx + i
        see = np.ones(L, dtype=bool)
        if causal:
            see &= j <= p
        if window > 0:
            see &= j > p - window
        if absent is not None:
            see &= ~absent
        if not see.any():
            continue
        for h in range(H):
            s = scale * (k[see, h // (H // Hk)] @ q[i, h])
            m = s.max()
            e = np.exp(s - m)
            out[i, h] = e @ v[see, h // (H // Hk)] / e.sum()
            lse[i, h] = m + np.log(e.sum())
    return out, lse
