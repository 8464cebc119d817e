"""The paged 4-bit key / value cache (pop_kv_plan, pop_kv_append, pop_kv_read, pop_kv_attention) against the numpy oracle.

Tolerances, derived before the first run.  Plans and codes are exact.  Attention is compared with 64-bit attention over
the values that the cache holds (so quantisation itself is no error):
  fp32   a dot product is split into bf16 pieces whose products are exact and summed in fp32 on the tensor cores; a step of those
         sums errs by at most 2^-21 + 2^-23 of its addends' magnitudes, D / 16 <= 8 steps, so a logit is off by at most
         2^-18 * scale * |q|_1 * max|k| =: dS.  Probabilities then err by 2 dS relative, and everything after by as many fp32 steps
         again on the values: |o - o_exact| <= (2 dS + 2^-17) max|v|.  In the 2-norm the signs average out: 1e-5.
  bf16   keys and values may pass through fp16 (11 bits; the group's mid point is rounded once, the value once more): 2^-10 of
         max|k| and max|v|, probabilities once to fp16 or a bf16 pair: 2^-11; the result is rounded to bf16: 2^-9 of itself.
         |o - o_exact| <= (2 * 2^-10 * scale * |q|_1 * max|k| + 2^-9) max|v| + 2^-9 |o|;  in the 2-norm 2.5e-3 (the rounding to
         bf16 alone has an rms of 1.7e-3).
"""
import ctypes as C
import subprocess
import sys

import numpy as np
import pytest
import torch

import __graft_entry__ as ge
from oracle import kv_oracle as ko
from paper_2602_06822_b200 import pop

F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _built():
    ge.build()
    pop.lib()


def i32(v):
    return torch.tensor(np.asarray(v, dtype=np.int32), device=DEV)


# ------------------------------------------------------------------------------------------------------------------ plan

def plan_case(rng, R, page, max_ctx, max_new, finished, spare, max_blocks=None):
    ctx = [int(x) for x in rng.integers(0, max_ctx + 1, R)]
    new = [int(x) for x in rng.integers(0, max_new + 1, R)]
    for r in range(R):
        if finished and r % finished == 1:
            new[r] = -1
    blocks = [-(-c // page) for c in ctx]
    need = sum(-(-(c + max(n, 0)) // page) - b for c, n, b in zip(ctx, new, blocks) if n >= 0)
    n_pages = max(1, sum(blocks) + need + spare)
    mb = max_blocks or max(1, max(-(-(c + max(n, 0)) // page) for c, n in zip(ctx, new)))
    perm = rng.permutation(n_pages)
    table = np.full((R, mb), -7, dtype=np.int32)
    at = 0
    for r, b in enumerate(blocks):
        b = min(b, mb)
        table[r, :b] = perm[at:at + b]
        at += b
    head = int(rng.integers(0, n_pages))
    count = n_pages - at
    ring = np.full(n_pages, -1, dtype=np.int32)
    ring[(head + np.arange(count)) % n_pages] = perm[at:]
    return ctx, new, table, ring, head, count


def check_plan(ctx, new, table, ring, head, count, page, capacity, in_place):
    want = ko.plan(ctx, new, table, ring, head, count, page, capacity)
    tb, rg, state = i32(table), i32(ring), i32([head, count])
    out = None if in_place else torch.full((2,), -1, dtype=torch.int32, device=DEV)
    p = pop.kv_plan(i32(ctx), i32(new), tb, rg, state, page, capacity, state_out=out)
    for name, got in (("table", tb), ("ring", rg), ("state", p.state), ("q_indptr", p.q_indptr), ("kv_lens", p.kv_lens),
                      ("slots", p.slots), ("positions", p.positions), ("info", p.info)):
        np.testing.assert_array_equal(got.cpu().numpy(), np.asarray(want[name]), err_msg=name)
    if not in_place:
        assert state.cpu().tolist() == [head, count]
    return want


@pytest.mark.gpu
@pytest.mark.parametrize("R,page,max_ctx,max_new,finished,spare", [
    (1, 16, 0, 1, 0, 0), (1, 16, 100, 0, 0, 3), (1, 64, 0, 5000, 0, 1), (8, 16, 1200, 1, 0, 9), (37, 32, 300, 40, 5, 0),
    (1023, 64, 500, 3, 7, 11), (1024, 128, 90, 1, 2, 0), (1025, 16, 33, 17, 3, 5), (4096, 64, 700, 30, 16, 1),
])
def test_plan_equals_the_oracle(R, page, max_ctx, max_new, finished, spare):
    rng = np.random.default_rng(R + page)
    case = plan_case(rng, R, page, max_ctx, max_new, finished, spare)
    total = sum(max(n, 0) for n in case[1])
    check_plan(*case, page, total, in_place=False)
    check_plan(*case, page, total + 5, in_place=True)
    if total > 2:
        check_plan(*case, page, total - 2, in_place=True)


@pytest.mark.gpu
@pytest.mark.parametrize("R", [5, 3000])
def test_plan_when_pages_run_out_or_the_row_is_full(R):
    rng = np.random.default_rng(R)
    ctx, new, table, ring, head, count = plan_case(rng, R, 16, 60, 40, 0, 0)
    short = max(0, count // 2)                      # half of the pages are gone
    want = check_plan(ctx, new, table, ring, head, short, 16, sum(new), in_place=False)
    assert want["info"][1] > 0 and -1 in want["slots"]
    ctx, new, table, ring, head, count = plan_case(rng, R, 16, 20, 60, 0, 50, max_blocks=3)
    want = check_plan(ctx, new, table, ring, head, count, 16, sum(new), in_place=True)
    assert -1 in want["slots"]


@pytest.mark.gpu
def test_plans_of_consecutive_steps_share_no_page():
    """Forty steps of a small server: requests grow, finish and start again; at every step the live pages and the free ones
    are a partition of all pages."""
    rng = np.random.default_rng(5)
    R, page, n_pages = 6, 16, 64
    table, ring, state = i32(np.full((R, 16), -1)), i32(np.arange(n_pages)), i32([0, n_pages])
    lens = np.zeros(R, dtype=np.int64)
    for step in range(40):
        new = rng.integers(0, 20, R)
        for r in range(R):
            if lens[r] + new[r] > 150 or (lens[r] > 0 and rng.random() < 0.1):
                new[r] = -1
        p = pop.kv_plan(i32(lens), i32(new), table, ring, state, page, int(np.maximum(new, 0).sum()))
        lens = np.where(new < 0, 0, lens + new)
        assert p.kv_lens.cpu().tolist() == lens.tolist() and p.info.cpu()[1] == 0
        t, (head, count) = table.cpu().numpy(), state.cpu().tolist()
        live = [int(x) for r in range(R) for x in t[r, :-(-int(lens[r]) // page)]]
        free = ring.cpu().numpy()[(head + np.arange(count)) % n_pages].tolist()
        assert sorted(live + free) == list(range(n_pages))


# ------------------------------------------------------------------------------------------------------- append and read

def filled(n_pages, page, heads, dim, value=255):
    pages = pop.kv_pages(n_pages, page, heads, dim, DEV)
    pages.fill_(value)
    return pages


def awkward_values(rng, T, H, D):
    x = rng.standard_normal((T, H, D)).astype(np.float32)
    x *= np.exp(rng.uniform(-6, 6, (T, H, 1))).astype(np.float32)
    x += (rng.standard_normal((1, H, D)) * (rng.random((1, H, D)) < 0.1) * 20).astype(np.float32)
    if T > 4:
        x[1] = 3.0                                   # one value throughout: scale 0
        x[2] = 0.0
        x[3, 0, ::3] = np.inf
        x[3, 0, 1::3] = np.nan
        x[4, 0, 5] = -np.inf
        x[4, -1] = np.linspace(0, 7.5, D)            # codes on ties
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,H,D,page,fused", [(1, 1, 64, 16, False), (3, 2, 128, 16, True), (17, 3, 64, 32, True), (64, 8, 128, 64, False),
                                              (150, 5, 128, 128, True), (333, 1, 64, 48, False)])
def test_append_and_read(T, H, D, page, fused, dtype):
    rng = np.random.default_rng(T + D)
    n_pages = -(-T // page) + 2
    slots = np.sort(rng.permutation(n_pages * page)[:T]) if T < 100 else rng.permutation(n_pages * page)[:T]
    kx, vx = (torch.from_numpy(awkward_values(rng, T, H, D)).to(dtype) for _ in range(2))
    if fused:
        rows = torch.zeros(T, 4, H, D, dtype=dtype, device=DEV)
        rows[:, 2], rows[:, 3] = kx.to(DEV), vx.to(DEV)
        kd, vd = rows[:, 2], rows[:, 3]
    else:
        kd, vd = kx.to(DEV), vx.to(DEV)
    pages = filled(n_pages, page, H, D)
    pop.kv_append(pages, kd, vd, torch.from_numpy(slots).to(DEV))
    raw = pages.cpu().numpy()
    want = [ko.stored(x.float().numpy()) for x in (kx, vx)]
    for i in rng.permutation(T)[:12]:                # byte for byte, by the format
        for h in range(H):
            got = ko.unpack_token(raw, int(slots[i]), h, D)
            np.testing.assert_array_equal(got[0], want[0][i, h])
            np.testing.assert_array_equal(got[1], want[1][i, h])
    free = np.setdiff1d(np.arange(n_pages * page), slots)
    G = D // 64
    for s in free[:20]:                              # nobody else's place was touched
        tile = raw[s // page, :, s % page // 16]
        assert (tile[:, G * 1024:].reshape(H, 16, -1)[:, s % 16] == 255).all()
    for out_dtype in (F32, BF16):
        k, v = pop.kv_read(pages, torch.from_numpy(slots).to(DEV), out_dtype)
        for got, w in ((k, want[0]), (v, want[1])):
            ref = torch.from_numpy(w).float().to(out_dtype)     # one rounding of the exact value to fp32 (then bf16)
            assert torch.equal(got.cpu(), ref)


@pytest.mark.gpu
def test_append_skips_slots_outside_the_cache_and_read_gives_zeros():
    pages = filled(2, 16, 2, 64)
    before = pages.clone()
    k = torch.randn(3, 2, 64, device=DEV)
    slots = torch.tensor([-1, 32, -5], device=DEV)
    pop.kv_append(pages, k, k, slots)
    assert torch.equal(pages, before)
    a, b = pop.kv_read(pages, slots, F32)
    assert float(a.abs().sum()) == 0.0 and float(b.abs().sum()) == 0.0
    pop.kv_append(pages, k[:0], k[:0], slots[:0])
    a, b = pop.kv_read(pages, slots[:0], BF16)
    assert a.shape == (0, 2, 64) and b.dtype == BF16


@pytest.mark.gpu
def test_quantisation_error_is_half_a_step():
    x = torch.randn(50, 4, 128, device=DEV)
    pages = filled(4, 16, 4, 128)
    slots = torch.arange(50, device=DEV)
    pop.kv_append(pages, x, x, slots)
    k, v = pop.kv_read(pages, slots, F32)
    g = x.unflatten(-1, (2, 64))
    step = (g.amax(-1) - g.amin(-1)) / 15
    # half a step, plus what rounding the scale and the zero point to fp16 moves (2^-11 of each, 15 steps at most)
    slack = step * (0.5 + 15 * 2.0 ** -11) + g.abs().amax(-1) * 2.0 ** -11
    for y in (k, v):
        assert ((y - x).unflatten(-1, (2, 64)).abs() <= slack[..., None] * (1 + 1e-5)).all()


# --------------------------------------------------------------------------------------------------------------- attention

class Setup:
    """Requests with lengths ctx + new in a paged cache, with the exact stored values beside it."""

    def __init__(self, seed, H, Hk, D, page, dtype, kv_lens, new, extra_pages=3, q_scale=1.5, pad_tokens=0, fused=False, first_page=0,
                 k_scale=1.0):
        rng = np.random.default_rng(seed)
        self.H, self.Hk, self.D, self.page, self.dtype = H, Hk, D, page, dtype
        self.kv_lens, self.new = [int(x) for x in kv_lens], [int(x) for x in new]
        R = len(kv_lens)
        blocks = [-(-n // page) for n in self.kv_lens]
        mb = max(1, max(blocks))
        n_pages = sum(blocks) + extra_pages
        perm = rng.permutation(n_pages) + first_page
        self.table = np.full((R, mb + 1), -1, dtype=np.int32)
        at = 0
        slots = []
        for r, b in enumerate(blocks):
            self.table[r, :b] = perm[at:at + b]
            at += b
            j = np.arange(self.kv_lens[r])
            slots.append(self.table[r, j // page].astype(np.int64) * page + j % page)
        slots = np.concatenate(slots)
        total = len(slots)

        def rnd(*shape):
            return torch.from_numpy(rng.standard_normal(shape).astype(np.float32))

        off = rnd(1, Hk, D) * 3 * torch.from_numpy((rng.random((1, Hk, D)) < 0.05).astype(np.float32))
        k, v = ((rnd(total, Hk, D) + off) * k_scale).to(dtype), rnd(total, Hk, D).to(dtype)
        self.k64, self.v64 = (ko.stored(x.float().numpy()) if total else np.zeros((0, Hk, D)) for x in (k, v))
        T = sum(self.new)
        q = (rnd(T + pad_tokens, H, D) * q_scale).to(dtype)
        self.q64 = q.double().numpy()
        if fused:
            rows = torch.zeros(T + pad_tokens, H + 2 * Hk, D, dtype=dtype, device=DEV)
            rows[:, :H] = q.to(DEV)
            self.q = rows[:, :H]
        else:
            self.q = q.to(DEV)
        self.pages = filled(n_pages + first_page, page, Hk, D)      # 0xff: NaN parameters wherever nothing is written
        if total:
            pop.kv_append(self.pages, k.to(DEV), v.to(DEV), torch.from_numpy(slots).to(DEV))
        self.indptr = np.concatenate([[0], np.cumsum(self.new)])
        self.T = T

    def run(self, **kw):
        return pop.kv_attention(self.pages, self.q, i32(self.table), i32(self.indptr), i32(self.kv_lens), **kw)

    def check(self, causal=True, window=0, scale=None, want_lse=True, rows=None, absent=None, **kw):
        lse = torch.full((self.q.shape[0], self.H), 7.0, device=DEV) if want_lse else None
        out = torch.full(self.q.shape, 7.0, dtype=self.dtype, device=DEV)
        self.run(causal=causal, window=window, scale=scale, out=out, lse_out=lse, **kw)
        sc = self.D ** -0.5 if scale is None else scale
        got, got_lse = out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()
        assert (got[self.T:] == 7.0).all()                           # padding tokens are left alone
        at, num, den = 0, 0.0, 0.0
        for r, (L, n) in enumerate(zip(self.kv_lens, self.new)):
            a, b = self.indptr[r], self.indptr[r + 1]
            k, v = self.k64[at:at + L], self.v64[at:at + L]
            at += L
            if n == 0:
                continue
            ab = None if absent is None else absent.get(r)
            o, l = ko.attention(self.q64[a:b], k, v, L - n, sc, causal, window, ab)
            g = got[a:b]
            empty = np.isneginf(l)
            assert (g[empty] == 0.0).all()
            if lse is not None:
                assert (np.isneginf(got_lse[a:b]) == empty).all()
            if L:
                kmax, vmax = np.abs(k).max(), np.abs(v).max()
                ds = abs(sc) * np.abs(self.q64[a:b]).sum(-1) * kmax          # [n, H]
                if self.dtype == F32:
                    tol = (2 * 2.0 ** -18 * ds + 2.0 ** -17) * vmax
                    tl = 2.0 ** -18 * ds + 2.0 ** -18
                else:
                    tol = (2 * 2.0 ** -10 * ds + 2.0 ** -9) * vmax
                    tl = 2.0 ** -10 * ds + 2.0 ** -18
                err = np.abs(g - o) - (2.0 ** -9 * np.abs(o) if self.dtype == BF16 else 0.0)
                assert (err <= tol[..., None]).all(), f"request {r} (kv {L}, new {n}): worst {np.max(err - tol[..., None]):.3e}"
                if lse is not None:
                    le = np.abs(got_lse[a:b] - l)[~empty]
                    assert (le <= (tl + 2.0 ** -20 * np.abs(np.where(empty, 0.0, l)))[~empty]).all()
            num += ((g - o) ** 2).sum()
            den += (o ** 2).sum()
        rel = np.sqrt(num / den) if den else 0.0
        assert rel <= (1e-5 if self.dtype == F32 else 2.5e-3), f"2-norm error {rel:.3e}"
        return out


HEADS = [(1, 1), (4, 4), (8, 2), (6, 2), (5, 1), (8, 1), (12, 1), (20, 1), (28, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", HEADS)
def test_single_tokens(heads, D, dtype):
    kv = [1, 0, 15, 16, 17, 63, 64, 65, 200, 33, 1, 500]
    new = [1, 1, 1, 1, 1, 1, 1, 1, 1, 0, 0, 1]
    for page in (16, 64):
        Setup(heads[0] + D, *heads, D, page, dtype, kv, new, fused=page == 64).check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 5), (True, 40), (False, 17), (True, 1)])
def test_masks(causal, window, dtype):
    # queries that stand before the first key (kv < new) see nothing; windows end inside tiles and pages
    kv = [3, 0, 40, 130, 16, 97, 300]
    new = [7, 2, 40, 3, 1, 50, 20]
    for H, Hk, D in ((4, 2, 64), (3, 1, 128)):
        Setup(window + 3, H, Hk, D, 32, dtype, kv, new).check(causal=causal, window=window)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,D", [((4, 4), 128), ((8, 2), 128), ((6, 2), 64), ((5, 1), 128), ((2, 2), 64)])
@pytest.mark.parametrize("kv,new", [([128], [128]), ([257], [257]), ([400, 70, 513], [129, 70, 300]), ([129, 1, 640, 0, 50], [1, 1, 383, 0, 33]),
                                    ([100, 300], [200, 290])])
def test_prompts(heads, D, kv, new, dtype):
    s = Setup(sum(kv), *heads, D, 64, dtype, kv, new, pad_tokens=3, fused=True)
    s.check()
    s.check(window=77)
    s.check(causal=False, want_lse=False)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_long_contexts_split_over_the_machine(dtype):
    Setup(1, 8, 2, 128, 64, dtype, [20011], [1]).check()
    Setup(2, 4, 4, 64, 128, dtype, [9000, 1, 333, 7777], [1, 1, 3, 2]).check()
    Setup(3, 2, 1, 128, 16, dtype, [12345], [1]).check(window=5000)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_short_requests(dtype):
    rng = np.random.default_rng(4)
    kv = rng.integers(0, 70, 700)
    Setup(4, 4, 2, 64, 16, dtype, kv, np.minimum(1, rng.integers(0, 5, 700))).check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sharp_and_flat_softmax(dtype):
    kv, new = [300, 150], [1, 150]
    s = Setup(8, 4, 2, 128, 64, dtype, kv, new, q_scale=20.0)          # one key takes nearly all
    s.check(scale=0.5 if dtype == F32 else None)
    s.check(scale=0.0)                                                 # all keys alike
    s.check(scale=-0.05)
    Setup(9, 4, 2, 128, 64, dtype, kv, new, q_scale=1e-6).check()
    Setup(10, 4, 2, 64, 64, dtype, kv, new, q_scale=3e4, k_scale=1e-4).check()


@pytest.mark.gpu
@pytest.mark.parametrize("new", [1, 60])
def test_nan_and_infinite_queries_stay_in_their_rows(new):
    for dtype in (BF16, F32):
        s = Setup(11, 4, 2, 128, 64, dtype, [200, 90], [new, 3])
        clean = s.run()
        s.q[0, 1, 5] = float("nan")
        s.q[new, 2, 7] = float("inf")
        out = s.run()
        assert torch.isnan(out[0, 1]).all()
        keep = torch.ones(out.shape[:2], dtype=torch.bool, device=DEV)
        keep[0, 1] = False
        keep[new, 2] = False
        assert torch.equal(out[keep], clean[keep]) and torch.isfinite(out[keep].float()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_missing_pages_are_not_seen(dtype):
    s = Setup(12, 4, 2, 64, 32, dtype, [200, 100, 64], [1, 100, 2])
    s.table[0, 2] = -1
    s.table[1, 0] = 10 ** 6
    s.table[2, :] = -1
    absent = {0: np.isin(np.arange(200) // 32, [2]), 1: np.arange(100) < 32, 2: np.ones(64, dtype=bool)}
    s.check(absent=absent)


@pytest.mark.gpu
def test_lengths_beyond_the_table_are_cut():
    s = Setup(13, 2, 2, 64, 16, BF16, [64, 40], [1, 1])
    want = s.run(causal=False)
    s.kv_lens = [10 ** 6, 40]
    s.table = np.ascontiguousarray(s.table[:, :4])
    assert torch.equal(s.run(causal=False), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_equal_calls_give_equal_bits_also_on_another_stream(dtype):
    s = Setup(14, 8, 2, 128, 64, dtype, [5000, 300, 2000, 17], [1, 200, 3, 17])
    a = s.run()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        b = s.run(stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(a, b) and torch.equal(a, s.run())


@pytest.mark.gpu
def test_offsets_past_32_bits():
    page, Hk, D = 128, 8, 128
    per_page = pop.kv_page_bytes(page, Hk, D)
    first = (1 << 32) // per_page + 9                                  # every page lies past 4 GiB
    for dtype, new in ((BF16, [1, 150]), (F32, [1, 20])):
        s = Setup(15, 16, 8, D, page, dtype, [700, 150], new, first_page=first)
        assert s.pages.numel() > 1 << 32
        s.check()
        slots = torch.tensor([int(s.table[0, 0]) * page + 5], device=DEV)
        k, _ = pop.kv_read(s.pages, slots, F32)
        assert torch.equal(k[0].cpu(), torch.from_numpy(s.k64[5]).float())
        del s
        torch.cuda.empty_cache()


@pytest.mark.gpu
def test_a_step_in_a_cuda_graph():
    """Plan, append and attention captured once and replayed: lengths live on the device, so the same graph serves every step."""
    torch.manual_seed(0)
    R, H, Hk, D, page, steps = 3, 8, 2, 128, 16, 20
    q, k, v = (torch.randn(steps, R, h, D, device=DEV).bfloat16() for h in (H, Hk, Hk))
    pages = filled(64, page, Hk, D)
    table, ring, state = i32(np.full((R, 8), -1)), i32(np.random.default_rng(1).permutation(64)), i32([0, 64])
    lens, ones = i32([0, 0, 0]), i32([1, 1, 1])
    qs, ks, vs = q[0].clone(), k[0].clone(), v[0].clone()

    def step():
        p = pop.kv_plan(lens, ones, table, ring, state, page, R)
        pop.kv_append(pages, ks, vs, p.slots)
        o = pop.kv_attention(pages, qs, table, p.q_indptr, p.kv_lens)
        lens.copy_(p.kv_lens)
        return o

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                                          # the workspace of this stream comes into being
        torch.cuda.synchronize()
        lens.zero_()
        table.fill_(-1)
        state.copy_(i32([0, 64]))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out = step()
    lens.zero_()
    table.fill_(-1)
    state.copy_(i32([0, 64]))
    for s in range(steps):
        qs.copy_(q[s]), ks.copy_(k[s]), vs.copy_(v[s])
        g.replay()
        torch.cuda.synchronize()
        k64, v64 = (ko.stored(x[:s + 1].float().cpu().numpy().reshape(-1, Hk, D)).reshape(s + 1, R, Hk, D) for x in (k, v))
        for r in range(R):
            want, _ = ko.attention(q[s, r:r + 1].double().cpu().numpy(), k64[:, r], v64[:, r], s, D ** -0.5, True, 0)
            got = out[r:r + 1].double().cpu().numpy()
            assert np.linalg.norm(got - want) <= 4e-3 * np.linalg.norm(want)       # one row: up to 2^-8 of it


# ---------------------------------------------------------------------------------------------------------------- refusals

def test_page_bytes():
    assert pop.kv_page_bytes(64, 8, 128) == 4 * 8 * 2304 and pop.kv_page_bytes(16, 1, 64) == 1152
    for args in ((64, 8, 96), (24, 8, 128), (2048, 8, 128)):
        with pytest.raises(pop.PopError) as e:
            pop.kv_page_bytes(*args)
        assert e.value.status == pop.POP_ERR_UNSUPPORTED
    with pytest.raises(pop.PopError) as e:
        pop.kv_page_bytes(0, 8, 128)
    assert e.value.status == pop.POP_ERR_INVALID_ARG


def _c_attention(**kw):
    """pop_kv_attention with addresses that are never followed: every call here is refused on the host."""
    a = dict(pages=1 << 20, n_pages=4, page_size=64, hk=2, dim=128, q=1 << 20, qs=512, dtype=pop.POP_BF16, heads=4, T=3, indptr=16, kv=16,
             R=2, table=16, mb=2, scale=0.1, causal=1, window=0, out=1 << 20, lse=None, ws=1 << 20, wsb=1 << 40)
    a.update(kw)
    d = pop.KVCacheDesc(a["pages"], a["n_pages"], a["page_size"], a["hk"], a["dim"])
    return pop.lib().pop_kv_attention(C.byref(d), a["q"], a["qs"], a["dtype"], a["heads"], a["T"], a["indptr"], a["kv"], a["R"], a["table"],
                                      a["mb"], a["scale"], a["causal"], a["window"], a["out"], a["lse"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw", [dict(pages=None), dict(pages=(1 << 20) + 8), dict(n_pages=0), dict(q=None), dict(q=(1 << 20) + 2), dict(qs=511),
                                dict(qs=508), dict(heads=5), dict(heads=0), dict(T=-1), dict(R=0), dict(mb=0), dict(window=-1), dict(out=None),
                                dict(ws=None), dict(wsb=1), dict(indptr=None), dict(kv=None), dict(table=None), dict(scale=float("nan")),
                                dict(out=(1 << 20) + 4)])
def test_attention_refuses_wrong_arguments(kw):
    assert _c_attention(**kw) == pop.POP_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [dict(dim=96), dict(dim=256), dict(page_size=24), dict(page_size=2048), dict(dtype=7),
                                dict(R=pop.POP_KV_MAX_REQUESTS + 1), dict(n_pages=1 << 30)])
def test_attention_refuses_what_it_does_not_take(kw):
    assert _c_attention(**kw) == pop.POP_ERR_UNSUPPORTED


def test_no_tokens_is_no_work():
    assert _c_attention(T=0, q=None, out=None) == pop.POP_OK


def test_append_read_and_plan_refuse_wrong_arguments():
    l = pop.lib()
    P = 1 << 20

    def desc(**kw):
        a = dict(pages=P, n=4, page=64, hk=2, dim=128)
        a.update(kw)
        return C.byref(pop.KVCacheDesc(a["pages"], a["n"], a["page"], a["hk"], a["dim"]))

    bad, no = pop.POP_ERR_INVALID_ARG, pop.POP_ERR_UNSUPPORTED
    assert l.pop_kv_append(None, P, 256, P, 256, 1, P, 3, None) == bad
    assert l.pop_kv_append(desc(), None, 256, P, 256, 1, P, 3, None) == bad
    assert l.pop_kv_append(desc(), P, 255, P, 256, 1, P, 3, None) == bad
    assert l.pop_kv_append(desc(), P, 256, P + 2, 256, 1, P, 3, None) == bad
    assert l.pop_kv_append(desc(), P, 256, P, 256, 1, None, 3, None) == bad
    assert l.pop_kv_append(desc(), P, 256, P, 256, 1, P, -1, None) == bad
    assert l.pop_kv_append(desc(dim=80), P, 256, P, 256, 1, P, 3, None) == no
    assert l.pop_kv_append(desc(), P, 256, P, 256, 5, P, 3, None) == no
    assert l.pop_kv_append(desc(), None, 0, None, 0, 1, None, 0, None) == pop.POP_OK
    assert l.pop_kv_read(desc(), P, 3, 1, None, P, None) == bad
    assert l.pop_kv_read(desc(page=17), P, 3, 1, P, P, None) == no
    assert l.pop_kv_attention_workspace(None) == bad and l.pop_kv_page_bytes(64, 8, 128, None) == bad
    good = [P, P, 4, 16, P, 8, P, P, P, 2, 4, P, P, P, None, None, None]
    for i in (0, 1, 4, 6, 7, 8, 11, 12, 13):
        args = list(good)
        args[i] = None
        assert l.pop_kv_plan(*args) == bad
    for i, v, rc in ((2, 0, bad), (2, 5000, no), (3, 20, no), (3, 0, bad), (5, 0, bad), (9, 0, bad), (10, -1, bad)):
        args = list(good)
        args[i] = v
        assert l.pop_kv_plan(*args) == rc


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(4, 4), (8, 2)])
@pytest.mark.parametrize("kv,new", [([0] * 70 + [300] + [9] * 89, [0] * 70 + [150] + [0] * 89),     # a prompt among requests without tokens
                                    ([200, 90, 33], [64, 1, 1]), ([200, 90, 33], [65, 1, 1]), ([200, 90, 33], [17, 0, 1]),
                                    ([200, 90, 0], [18, 0, 0]), ([64], [16]), ([65], [17])])
def test_lengths_at_which_kernels_change(kv, new, heads):
    Setup(len(kv) + sum(new), *heads, 64, 16, BF16, kv, new).check()


@pytest.mark.gpu
def test_check_reports_a_wait_that_ran_out_and_clears_it():
    """The status word as a kernel that gives up would leave it (set from the host: no kernel is made to give up)."""
    s = Setup(21, 4, 2, 64, 16, BF16, [150, 20], [150, 1])
    n = C.c_size_t()
    assert pop.lib().pop_kv_attention_workspace(C.byref(n)) == pop.POP_OK
    ws = torch.zeros(n.value, dtype=torch.uint8, device=DEV)
    want = s.run(workspace=ws)
    pop.kv_attention_check(DEV, workspace=ws)
    ws[0] = 1
    with pytest.raises(pop.PopError) as e:
        pop.kv_attention_check(DEV, workspace=ws)
    assert e.value.status == pop.POP_ERR_TIMEOUT
    pop.kv_attention_check(DEV, workspace=ws)
    assert torch.equal(s.run(workspace=ws), want)                      # usable afterwards
    pop.kv_attention_check(DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("T,H,requests", [(40, 3, 1), (1200, 8, 3), (2100, 8, 700)])
def test_append_of_runs_that_begin_anywhere(T, H, requests):
    """Whole tiles, parts of tiles and single tokens in one call, and skipped tokens among them; few and many tokens."""
    rng = np.random.default_rng(T)
    page, D = 32, 128
    cut = np.sort(rng.choice(np.arange(1, T), requests - 1, replace=False)) if requests > 1 else []
    new = np.diff(np.concatenate([[0], cut, [T]])).astype(int)
    ctx = rng.integers(0, 70, requests)
    blocks = [-(-int(c + n) // page) for c, n in zip(ctx, new)]
    perm, at, slots = rng.permutation(sum(blocks)), 0, []
    for c, n, b in zip(ctx, new, blocks):
        j = np.arange(c, c + n)
        slots.append(perm[at:at + b][j // page] * page + j % page)
        at += b
    slots = np.concatenate(slots)
    skip = rng.random(T) < 0.02
    pages = filled(sum(blocks), page, H, D)
    for dtype in (BF16, F32):
        k, v = (torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32)).to(dtype) for _ in range(2))
        given = torch.from_numpy(np.where(skip, -1, slots)).to(DEV)
        pop.kv_append(pages, k.to(DEV), v.to(DEV), given)
        a, b = pop.kv_read(pages, given, F32)
        for x, y in ((k, a), (v, b)):
            want = ko.stored(x.float().numpy()).astype(np.float32)
            want[skip] = 0
            np.testing.assert_array_equal(y.cpu().numpy(), want)


@pytest.mark.gpu
def test_binding_refuses_wrong_tensors():
    pages = filled(4, 16, 2, 64)
    k = torch.randn(3, 2, 64, device=DEV)
    slots = torch.arange(3, device=DEV)
    for bad in (lambda: pop.kv_append(pages, k, k[:2], slots), lambda: pop.kv_append(pages, k[:, :1], k, slots),
                lambda: pop.kv_append(pages, k, k, slots.int()), lambda: pop.kv_append(pages[:, :, :, ::2], k, k, slots),
                lambda: pop.kv_append(pages, k.transpose(0, 1).contiguous().transpose(0, 1), k, slots),
                lambda: pop.kv_append(pages, k, k, slots.cpu()), lambda: pop.kv_read(pages, slots.view(1, 3), F32),
                lambda: pop.kv_attention(pages, k, i32([[0]]), i32([0, 3, 3]), i32([3])),
                lambda: pop.kv_attention(pages, k, i32([[0]]), i32([0, 3]), i32([3]), out=k.bfloat16()),
                lambda: pop.kv_attention(pages, k, i32([[0]]), i32([0, 3]), i32([3]), lse_out=k)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: pop.kv_append(pages, k.half(), k.half(), slots), lambda: pop.kv_append(pages, k, k.bfloat16(), slots),
                lambda: pop.kv_read(pages, slots, torch.float16)):
        with pytest.raises(TypeError):
            bad()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 8, 2 ** 30, 2 ** 33])
def test_a_window_beyond_every_length_hides_nothing(window, dtype):
    """Row blocks of the streaming kernel (fp32, and bf16 requests of 17 to 64 rows), prompts, queries before the first key."""
    s = Setup(22, 4, 2, 64, 16, dtype, [300, 90, 40, 5, 700], [150, 9, 30, 32, 1])
    for causal in (True, False):
        assert torch.equal(s.run(causal=causal, window=window), s.run(causal=causal, window=0))
    s.check(window=window)


@pytest.mark.gpu
def test_negative_windows_are_refused():
    s = Setup(23, 2, 2, 64, 16, BF16, [20], [1])
    for window in (-1, -2 ** 31, -2 ** 32 - 5):
        with pytest.raises(pop.PopError) as e:
            s.run(window=window)
        assert e.value.status == pop.POP_ERR_INVALID_ARG


FULL_ROWS = [     # ctx, new, max_blocks, free pages -> state, info, what each row has then (pages of 16 tokens, free ones 100, 101, ..)
    ([0], [80], 3, 10, [3, 7], [80, 2], [[100, 101, 102]]),
    ([32], [64], 2, 6, [0, 6], [64, 4], [[0, 1]]),
    ([60, 5], [40, 30], 2, 4, [1, 3], [70, 4], [[0, 1], [2, 100]]),
    ([0, 20, 0], [70, 40, 20], 3, 5, [5, 0], [130, 4], [[100, 101, 102], [0, 1, 103], [104, -1, -7]]),
]


def full_row_case(ctx, new, max_blocks, free):
    table, at = np.full((len(ctx), max_blocks), -7, dtype=np.int32), 0
    for r, c in enumerate(ctx):
        n = min(-(-c // 16), max_blocks)
        table[r, :n] = range(at, at + n)
        at += n
    ring = np.full(110, -1, dtype=np.int32)
    ring[:free] = range(100, 100 + free)
    return table, ring


@pytest.mark.parametrize("ctx,new,max_blocks,free,state,info,rows", FULL_ROWS)
def test_oracle_gives_a_full_row_no_pages(ctx, new, max_blocks, free, state, info, rows):
    table, ring = full_row_case(ctx, new, max_blocks, free)
    w = ko.plan(ctx, new, table, ring, 0, free, 16, sum(new))
    assert w["state"] == state and w["info"] == info and w["table"].tolist() == rows
    lost = sum(max(0, c + n - max(c, max_blocks * 16)) for c, n in zip(ctx, new))
    assert w["slots"].count(-1) >= lost


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("ctx,new,max_blocks,free,state,info,rows", FULL_ROWS)
def test_a_full_row_takes_no_pages_from_the_ring(ctx, new, max_blocks, free, state, info, rows, in_place):
    table, ring = full_row_case(ctx, new, max_blocks, free)
    w = check_plan(ctx, new, table, ring, 0, free, 16, sum(new), in_place)
    assert w["state"] == state and w["info"] == info


@pytest.mark.gpu
def test_many_full_rows_among_others():
    rng = np.random.default_rng(31)
    for R in (900, 4096):
        ctx, new, table, ring, head, count = plan_case(rng, R, 16, 20, 60, 7, 50, max_blocks=3)
        for in_place in (True, False):
            w = check_plan(ctx, new, table, ring, head, count, 16, sum(max(n, 0) for n in new), in_place)
            over = sum(-(-(c + n) // 16) - max(3, -(-c // 16)) for c, n in zip(ctx, new) if n >= 0 and c + n > 48)
            assert w["info"][1] == over > 0


def short_of_pages(plan, steps, seed):
    """A server with fewer pages than its requests want and rows that they outgrow: some are refused pages, finish, and start again.  After
    every step the pages in the live rows and the free ones are all pages, each once."""
    rng = np.random.default_rng(seed)
    R, page, mb, n_pages = 7, 16, 6, 20
    table, ring, head, count = np.full((R, mb), -1, dtype=np.int32), rng.permutation(n_pages).astype(np.int32), 3, n_pages
    lens, refused, holes = np.zeros(R, dtype=np.int64), 0, 0
    for _ in range(steps):
        new = rng.integers(0, 50, R)
        new[(lens > 0) & (rng.random(R) < 0.25)] = -1
        for r in np.flatnonzero(new < 0):
            holes += int((table[r, :min(mb, -(-lens[r] // page))] < 0).sum())
        w = plan(lens.tolist(), new.tolist(), table, ring, head, count, page)
        table, ring, (head, count) = np.asarray(w["table"]), np.asarray(w["ring"]), w["state"]
        lens = np.asarray(w["kv_lens"])
        refused += w["info"][1]
        rows = np.concatenate([table[r, :min(mb, -(-int(n) // page))] for r, n in enumerate(lens)])
        free = ring[(head + np.arange(count)) % n_pages]
        assert sorted(rows[rows >= 0].tolist() + free.tolist()) == list(range(n_pages))
        assert w["slots"].count(-1) == 0 or refused
    assert refused > 0 and holes > 0


@pytest.mark.parametrize("seed", [0, 1])
def test_oracle_recovers_from_running_out_of_pages(seed):
    short_of_pages(lambda c, n, t, r, h, k, page: ko.plan(c, n, t, r, h, k, page, sum(max(x, 0) for x in n)), 60, seed)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [True, False])
def test_pages_run_out_and_come_back(in_place):
    short_of_pages(lambda c, n, t, r, h, k, page: check_plan(c, n, t, r, h, k, page, sum(max(x, 0) for x in n), in_place), 60, 2)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("R,max_ctx", [(40, 900), (4000, 500)])
def test_finished_rows_with_entries_that_are_no_page(R, max_ctx, in_place):
    """Also more entries than are given back at a time (4096)."""
    rng = np.random.default_rng(R)
    ctx, new, table, ring, head, count = plan_case(rng, R, 16, max_ctx, 20, 2, 5)
    hole = rng.random(table.shape) < 0.2
    table[hole] = np.where(rng.random(int(hole.sum())) < 0.5, -1, 10 ** 6)
    gone = [int(p) for r in range(R) if new[r] < 0 for p in table[r, :-(-ctx[r] // 16)]]
    assert len(gone) > (4096 if R > 1000 else 100)
    w = check_plan(ctx, new, table, ring, head, count, 16, sum(max(n, 0) for n in new), in_place)
    assert w["state"][1] == count + sum(0 <= p < len(ring) for p in gone) - (w["state"][0] - head) % len(ring)


@pytest.mark.gpu
@pytest.mark.parametrize("R", [4000, 4063, 4064, 4095])
def test_plans_of_nearly_the_most_requests_as_a_process_first_call(R):
    """(A larger call before would have asked for the shared memory that these need, so each has a process of its own.)"""
    code = f"""
import torch
from paper_2602_06822_b200 import pop
R, kw = {R}, dict(dtype=torch.int32, device="cuda")
table = torch.full((R, 2), -1, **kw)
p = pop.kv_plan(torch.zeros(R, **kw), torch.ones(R, **kw), table, torch.arange(R + 3, **kw), torch.tensor([0, R + 3], **kw), 16, R)
assert p.q_indptr.tolist() == list(range(R + 1)) and p.slots.tolist() == list(range(0, 16 * R, 16))
assert table[:, 0].tolist() == list(range(R)) and p.state.tolist() == [R, 3] and p.info.tolist() == [R, 0]
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=ge.ROOT, timeout=300)


# Values that the cache holds are finite (infinities count as +-65504), but with the rounding of scale and zero point a group's top code can
# stand for up to 65536, which fp16 has no finite number for.  Each row: what is put at dimensions 5 and 70 of a row of ordinary values, or
# the whole row.
def saturated_rows(rng, Hk, D):
    rows = []
    for a, b in ((np.inf, 1.0), (np.inf, -np.inf), (-np.inf, np.inf), (65504.0, 65504.0), (-65504.0, 7e4), (65280.0, 0.0), (3e38, 3.0)):
        x = rng.standard_normal((Hk, D)).astype(np.float32)
        x[:, 5], x[:, D - 58] = a, b                              # (D = 64: dimensions 5 and 6 of one group)
        rows.append(x)
    both = rng.standard_normal((Hk, D)).astype(np.float32)
    both[:, ::9], both[:, 1::9] = np.inf, -np.inf
    rows += [both, np.full((Hk, D), np.inf, dtype=np.float32), np.full((Hk, D), -np.inf, dtype=np.float32)]
    for lo, hi in ((-65504.0, -65414.0), (65400.0, 65504.0), (0.0, 65504.0), (1.0, 65504.0), (-34814.0, 65504.0), (3e4, 65504.0)):
        rows.append(np.linspace(lo, hi, D, dtype=np.float32)[None].repeat(Hk, 0))
    return rows


def put(s, r, j, k, v):
    """Key and value [Hk, D] (fp32, of s's type) as token j of request r, in the cache and in the exact values beside it."""
    k, v = (torch.from_numpy(x)[None].to(s.dtype) for x in (k, v))
    slot = int(s.table[r, j // s.page]) * s.page + j % s.page
    pop.kv_append(s.pages, k.to(DEV), v.to(DEV), torch.tensor([slot], device=DEV))
    at = sum(s.kv_lens[:r]) + j
    s.k64[at], s.v64[at] = (ko.stored(x.float().numpy())[0] for x in (k, v))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_reads_saturated_values_as_finite(D, dtype):
    """One key, so that the output is its value.  bf16: one of the two numbers next to it (it is rounded to fp16, or limited to 65504,
    and then to bf16).  fp32: three bf16 pieces and the sums of its group's codes."""
    rng = np.random.default_rng(41)
    rows = saturated_rows(rng, 2, D)
    one = Setup(41, 4, 2, D, 16, dtype, [1] * len(rows), [1] * len(rows))
    many = [Setup(42 + i, 4, 2, D, 16, dtype, [1], [70]) for i in range(len(rows))]
    for i, x in enumerate(rows):
        put(one, i, 0, one.k64[i].astype(np.float32), x)
        put(many[i], 0, 0, many[i].k64[0].astype(np.float32), x)
    got = [one.run(causal=False).double().cpu().numpy()[:, None]]
    got += [np.stack([m.run(causal=False).double().cpu().numpy() for m in many])]
    want = one.v64.repeat(2, 1)                                    # [request, heads, D]
    group = np.abs(want).reshape(len(rows), 4, -1, 64).max(-1, keepdims=True).repeat(64, -1).reshape(want.shape)
    size = np.abs(want).astype(np.float32).view(np.uint32)
    below, above = (((size >> 16) + i << 16).astype(np.uint32).view(np.float32).astype(np.float64) for i in (0, 1))
    for g in got:
        assert np.isfinite(g).all()
        if dtype == BF16:
            assert (((np.abs(g) == below[:, None]) | (np.abs(g) == above[:, None])) & (g * want[:, None] >= 0)).all()
        else:
            assert (np.abs(g - want[:, None]) <= (2.0 ** -18 * (np.abs(want) + group))[:, None]).all()


def near_in_every_element(s, **mask):
    """bf16 attention, element by element (a 2-norm would be that of the few elements that are large).  Keys may be rounded to fp16: a logit is
    off by 2^-11 of ds = scale |q|_1 max|k|, a weight by twice that and its own 2^-11; a value by 2^-11, or 2^-11 where it is limited;
    the result by 2^-8, half a unit of bf16."""
    got = s.run(**mask).double().cpu().numpy()
    at = 0
    for r, (L, n) in enumerate(zip(s.kv_lens, s.new)):
        a, b = s.indptr[r], s.indptr[r + 1]
        q, k, v = s.q64[a:b], s.k64[at:at + L], s.v64[at:at + L]
        o, size = (ko.attention(q, k, x, L - n, s.D ** -0.5, mask.get("causal", True), mask.get("window", 0))[0] for x in (v, np.abs(v)))
        ds = s.D ** -0.5 * np.abs(q).sum(-1, keepdims=True) * np.abs(k).max()
        off = (2 * 2.0 ** -11 * ds + 3 * 2.0 ** -11) * size
        assert (np.abs(got[a:b] - o) <= off + 2.0 ** -8 * (np.abs(o) + off)).all()
        at += L


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kv,new", [([150], [9]), ([150], [70]), ([400, 150], [1, 100]), ([90, 150], [1, 12])])
def test_saturated_tokens_that_are_hidden_change_nothing(kv, new, D, dtype):
    """The last request's token 141: queries that do not see it (causal, window) have the bits that they have with an ordinary one there,
    those that do are near the exact result."""
    rng = np.random.default_rng(43)
    r, j = len(kv) - 1, 141
    first = sum(new[:r])
    masks = [dict(causal=True), dict(causal=True, window=3), dict(causal=False, window=4)]
    s = Setup(43, 4, 2, D, 32, dtype, kv, new)
    clean = [s.run(**m) for m in masks]
    k0, v0 = (x[sum(kv[:r]) + j].astype(np.float32) for x in (s.k64, s.v64))
    pos = torch.arange(new[r], device=DEV) + kv[r] - new[r]
    hidden = [pos < j, (pos < j) | (pos - j >= 3), pos - j >= 4]
    for x in saturated_rows(rng, 2, D):
        for key, value in ((k0, x), (x, v0), (x, x)):
            put(s, r, j, key, value)
            for m, c, h in zip(masks, clean, hidden):
                out = s.run(**m)
                assert torch.isfinite(out.float()).all()
                assert torch.equal(out[:first], c[:first]) and torch.equal(out[first:][h], c[first:][h])
        put(s, r, j, k0, x)
        for m in masks:
            if dtype == F32:
                s.check(want_lse=False, **m)
            else:
                near_in_every_element(s, **m)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kv,new", [([600], [1]), ([600, 40], [5, 1]), ([600], [90])])
def test_saturated_tokens_all_over_the_context(kv, new, D):
    rng = np.random.default_rng(44)
    s = Setup(44, 8, 2, D, 64, BF16, kv, new)
    rows = saturated_rows(rng, 2, D)
    for i, j in enumerate([*range(0, 590, 37), 64, 65, 100, 101]):
        put(s, 0, j, s.k64[j].astype(np.float32), rows[i % len(rows)])
    near_in_every_element(s)
    near_in_every_element(s, window=50)
    near_in_every_element(s, causal=False)


def calls_of_every_kind(pages, k, slots, ctx, table, ring, state, indptr, stream=None):
    """(which argument, call without it): the calls of the binding with one tensor given from outside."""
    plan = dict(ctx_lens=ctx, new_lens=ctx, block_table=table, ring=ring, state=state, state_out=state.clone())
    attend = dict(pages=pages, q=k, block_table=table, q_indptr=indptr, kv_lens=ctx, out=k.clone(),
                  lse_out=torch.zeros(k.shape[:2], device=DEV), workspace=torch.zeros(16 << 20, dtype=torch.uint8, device=DEV))
    for name, t in plan.items():
        yield name, t, lambda x, name=name: pop.kv_plan(**{**plan, name: x}, page_size=16, n_tokens=1, stream=stream)
    for name, t in (("pages", pages), ("k", k), ("v", k), ("slots", slots)):
        yield name, t, lambda x, name=name: pop.kv_append(**{**dict(pages=pages, k=k, v=k, slots=slots), name: x}, stream=stream)
    for name, t in (("pages", pages), ("slots", slots)):
        yield name, t, lambda x, name=name: pop.kv_read(**{**dict(pages=pages, slots=slots), name: x}, dtype=F32, stream=stream)
    for name, t in attend.items():
        yield name, t, lambda x, name=name: pop.kv_attention(**{**attend, name: x}, stream=stream)


def small_arguments():
    ctx = i32([1, 1])
    return (filled(4, 16, 2, 64), torch.randn(2, 2, 64, device=DEV), torch.arange(2, device=DEV), ctx, i32([[0], [1]]), i32([2, 3, 0, 0]),
            i32([0, 2]), i32([0, 1, 2]))


@pytest.mark.gpu
def test_host_tensors_are_refused():
    """One of them on the host, and all of a plan's (which would then be on one device, but not on this one)."""
    for name, t, call in calls_of_every_kind(*small_arguments()):
        with pytest.raises(ValueError):
            call(t.cpu())
    ctx, table, ring, state = (x.cpu() for x in (i32([1, 1]), i32([[0], [1]]), i32([2, 3, 0, 0]), i32([0, 2])))
    with pytest.raises(ValueError):
        pop.kv_plan(ctx, ctx, table, ring, state, 16, 2)


@pytest.mark.gpu
def test_tensors_of_another_device_than_the_current_one_are_refused(monkeypatch):
    args = small_arguments()
    calls = list(calls_of_every_kind(*args))
    cache = pop.KVCache(1, 1, 32, 2, 64)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)                 # as if another one were current: nothing may be launched
    before = pop.kernel_launch_count()
    for name, t, call in calls:
        with pytest.raises(ValueError):
            call(t)
    with pytest.raises(ValueError):
        cache.plan(i32([1]), 1)
    assert pop.kernel_launch_count() == before


@pytest.mark.gpu
def test_a_stream_of_another_device_is_refused():
    class Elsewhere:
        device_index, cuda_stream = 1, 0
    for name, t, call in calls_of_every_kind(*small_arguments(), stream=Elsewhere()):
        with pytest.raises(ValueError):
            call(t)


@pytest.mark.gpu
def test_tensors_that_require_a_gradient_are_refused():
    pages, k, slots, ctx, table, _, _, indptr = small_arguments()
    x = k.clone().requires_grad_()
    for call in (lambda: pop.kv_append(pages, x, k, slots), lambda: pop.kv_append(pages, k, x * 2, slots),
                 lambda: pop.kv_attention(pages, x, table, indptr, ctx)):
        with pytest.raises(ValueError, match="backward"):
            call()
    with torch.no_grad():
        pop.kv_append(pages, x, x, slots * 16)                       # (each request's first token)
        want = pop.kv_attention(pages, x, table, indptr, ctx)
    assert torch.equal(pop.kv_attention(pages, x.detach(), table, indptr, ctx), want)
