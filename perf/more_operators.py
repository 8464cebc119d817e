"""What the operators around a decoder layer's attention are measured on: the norms before and after a block with its gate and
its residual addition, rotary positions (alone, and on the way into the 4-bit key/value cache), and the matrix product in
8-bit floating point with a scale for every block of 128; with a plain form of each in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 128                 # elements (along the summed dimension) that share a scale; 128 x 128 for weights
E4M3_MAX = 448.0
EPS = 1e-5


# ------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one token of the decoder: the residual addition after the attention block and the norm before the FFN; pure latency
        dict(name="norm_decode", op="norm", tokens=1, d=4096, dtype="bf16", post=False, gate="none", scaled=False),
        # a small fp32 model of an odd width, the block's output normalised and gated by channel
        dict(name="norm_f32", op="norm", tokens=517, d=1001, dtype="f32", post=True, gate="channel", scaled=True),
        # many prompts at once, norms on both sides of the block and a gate for every token
        dict(name="norm_prompt", op="norm", tokens=16384, d=4096, dtype="bf16", post=True, gate="token", scaled=True),
        # a decode step of a small batch, grouped heads, far positions: q rotated, k rotated and written to the cache with v
        dict(name="rope_decode", op="rope", tokens=13, requests=13, heads=32, kv_heads=8, dim=128, rot=128, interleaved=False,
             scaling="none", factor=1.0, far=100000, dtype="bf16", cache=True, page=64, fused=True),
        # a ragged fp32 batch, a quarter of the head in neighbouring pairs, positions scaled for a long context
        dict(name="rope_f32", op="rope", tokens=517, requests=5, heads=12, kv_heads=4, dim=96, rot=24, interleaved=True,
             scaling="yarn", factor=16.0, far=60000, dtype="f32", cache=False, page=0, fused=False),
        # many prompts at once into the cache, out of the rows of one projection
        dict(name="rope_prompt", op="rope", tokens=16384, requests=24, heads=32, kv_heads=8, dim=128, rot=128, interleaved=False,
             scaling="none", factor=1.0, far=0, dtype="bf16", cache=True, page=64, fused=True),
        # one token through the decoder's three attention projections as one
        dict(name="linear_decode", op="linear", tokens=1, n=12288, k=4096, dtype="bf16", norm=False),
        # the same for a small batch, behind the norm that feeds it
        dict(name="linear_after_norm", op="linear", tokens=13, n=12288, k=4096, dtype="bf16", norm=True),
        # a small fp32 model's prompt, sizes that fill no tile
        dict(name="linear_f32", op="linear", tokens=333, n=1000, k=1360, dtype="f32", norm=False),
        # a large decode batch (or a short prompt) through the output projection
        dict(name="linear_chunk", op="linear", tokens=100, n=4096, k=4096, dtype="bf16", norm=False),
        # the decoder's prompt of 1024 tokens
        dict(name="linear_prompt", op="linear", tokens=1024, n=12288, k=4096, dtype="bf16", norm=False),
        # many prompts at once through a down projection
        dict(name="linear_bulk", op="linear", tokens=16384, n=4096, k=11008, dtype="bf16", norm=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: a norm, a rotation or a product of the listed ones' ranges."""
    op = rng.choice(("norm", "rope", "linear", "linear"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "norm":
        d = rng.choice((_log_int(rng, 33, 8192), 8 * _log_int(rng, 8, 1024)))
        return dict(op="norm", tokens=_log_int(rng, 1, min(16384, 16384 * 4096 // d // (2 if dtype == "f32" else 1))), d=d, dtype=dtype,
                    post=rng.choice((True, False)), gate=rng.choice(("none", "channel", "token")), scaled=rng.choice((True, False)))
    if op == "rope":
        cache = rng.choice((True, False))
        dim = rng.choice((64, 128, 128)) if cache else rng.choice((64, 80, 96, 128, 192, 256))
        kv_heads = rng.choice((1, 2, 3, 4, 8))
        heads = kv_heads * rng.choice((1, 2, 3, 4, 8))
        requests = _log_int(rng, 1, 64)
        most = max(64, 16384 * 48 * 128 // ((heads + 2 * kv_heads) * dim) // (2 if dtype == "f32" else 1))
        return dict(op="rope", tokens=max(requests, _log_int(rng, 1, min(16384, most))), requests=requests, heads=heads, kv_heads=kv_heads,
                    dim=dim, rot=rng.choice((dim, dim, dim // 2, dim // 4)), interleaved=rng.choice((True, False)),
                    scaling=rng.choice(("none", "linear", "ntk", "yarn", "bands")), factor=rng.choice((2.0, 8.0, 16.0)),
                    far=rng.choice((0, _log_int(rng, 100, 120000))), dtype=dtype, cache=cache, page=rng.choice((16, 32, 64, 128)) if cache else 0,
                    fused=rng.choice((True, False)))
    n, k = _log_int(rng, 64, 14336), 16 * _log_int(rng, 4, 896)
    tokens = _log_int(rng, 1, max(1, min(16384, 16384 * 4096 * 11008 // (n * k) // (2 if dtype == "f32" else 1))))
    return dict(op="linear", tokens=tokens, n=n, k=k, dtype=dtype, norm=rng.choice((True, False, False)) and dtype == "bf16")


# ----------------------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed % (1 << 62))
    return g


def _stream(tokens, d, g):
    """A residual stream: a few channels far larger than the others, tokens of different size."""
    x = torch.randn(tokens, d, generator=g, device=DEV)
    big = torch.rand(d, generator=g, device=DEV) < 0.01
    x = torch.where(big, x * 12, x)
    return x * torch.exp(0.5 * torch.randn(tokens, 1, generator=g, device=DEV))


def _gain(d, g):
    return 1 + 0.2 * torch.randn(d, generator=g, device=DEV)


def _norm_inputs(case, seed):
    """h, the block's output, its gain and gate, the gain of the norm that follows."""
    T, d, dt, g = case["tokens"], case["d"], DTYPES[case["dtype"]], _generator(seed)
    h, u = _stream(T, d, g).to(dt), (0.7 * torch.randn(T, d, generator=g, device=DEV)).to(dt)
    post = _gain(d, g).to(dt) if case["post"] else None
    gate = None
    if case["gate"] != "none":
        gate = torch.sigmoid(torch.randn(T if case["gate"] == "token" else 1, d, generator=g, device=DEV)).to(dt)
    return h, u, post, gate, _gain(d, g).to(dt)


def _scales(case):
    return (0.9, 0.35) if case["scaled"] else (1.0, 1.0)


def _shares(case):
    """Tokens of each request of a rope case (near-equal ragged shares) and where in the request they start."""
    n, t = case["requests"], case["tokens"]
    cut = [0]
    for i in range(1, n):
        cut.append(min(t - (n - i), max(cut[-1] + 1, round(t * i / n) + (7 * i) % 5 - 2)))
    cut.append(t)
    new = [b - a for a, b in zip(cut, cut[1:])]
    return [(37 * i) % 150 for i in range(n)], new


def _rope_inputs(case, seed):
    """q, k, v rows and the tokens' positions."""
    T, H, Hk, D, dt, g = case["tokens"], case["heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]], _generator(seed)
    rows = torch.randn(T, H + 2 * Hk, D, generator=g, device=DEV)
    rows[:, H:H + Hk] += 3 * torch.randn(Hk, D, generator=g, device=DEV) * (torch.rand(Hk, D, generator=g, device=DEV) < 0.05)
    rows = rows.to(dt)
    q, k, v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    if not case["fused"]:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    ctx, new = _shares(case)
    pos = np.concatenate([np.arange(c, c + n) for c, n in zip(ctx, new)]) + (case["far"] + int(seed) % 97 if case["far"] else 0)
    return q, k, v, torch.from_numpy(pos).to(DEV, torch.int32)


def _linear_inputs(case, seed):
    """The rows that the product (or the norm before it) takes, and the weights' codes and scales."""
    T, N, K, dt, g = case["tokens"], case["n"], case["k"], DTYPES[case["dtype"]], _generator(seed)
    x = _stream(T, K, g).to(dt)
    u = (0.7 * torch.randn(T, K, generator=g, device=DEV)).to(dt) if case["norm"] else None
    gain = _gain(K, g).to(dt) if case["norm"] else None
    w = 0.02 * torch.randn(N, K, generator=g, device=DEV) * torch.exp(0.3 * torch.randn(N, 1, generator=g, device=DEV))
    nb, kb = -(-N // BLOCK), -(-K // BLOCK)
    padded = torch.zeros(nb * BLOCK, kb * BLOCK, device=DEV)
    padded[:N, :K] = w
    blocks = padded.view(nb, BLOCK, kb, BLOCK)
    scales = (blocks.abs().amax((1, 3)) * (1.0 / E4M3_MAX)).clamp(min=2.0 ** -126)
    codes = (blocks * (1.0 / scales)[:, None, :, None]).clamp(-E4M3_MAX, E4M3_MAX).view(nb * BLOCK, kb * BLOCK)[:N, :K]
    return x, u, gain, codes.to(torch.float8_e4m3fn).contiguous(), scales.contiguous()


def prepare(case, seed):
    if case["op"] == "norm":
        h, u, post, gate, gain = _norm_inputs(case, seed)
        return dict(case=case, h=h, u=u, post=post, gate=gate, gain=gain)
    if case["op"] == "linear":
        x, u, gain, codes, scales = _linear_inputs(case, seed)
        return dict(case=case, x=x, u=u, gain=gain, codes=codes, scales=scales)
    q, k, v, pos = _rope_inputs(case, seed)
    st = dict(case=case, q=q, k=k, v=v, pos=pos)
    if case["cache"]:
        ctx, new = _shares(case)
        page = case["page"]
        blocks = [-(-(c + n) // page) for c, n in zip(ctx, new)]
        n_pages = sum(blocks) + 3
        perm = np.random.RandomState((seed * 31 + 5) % (1 << 31)).permutation(n_pages)
        first = np.cumsum([0] + blocks)
        slots = [perm[first[r] + np.arange(c, c + n) // page] * page + np.arange(c, c + n) % page for r, (c, n) in enumerate(zip(ctx, new))]
        st["slots"] = torch.from_numpy(np.concatenate(slots).astype(np.int64)).to(DEV)
        tile = case["dim"] // 64 * (2 * 512 + 16 * 8)                        # bytes of 16 tokens of one head in 4 bits
        st["pages"] = torch.full((n_pages, case["kv_heads"], page // 16, tile), 255, dtype=torch.uint8, device=DEV)
    if own:                                                                  # the table of frequencies that a program keeps
        from paper_2602_06822_b200 import pop
        st["rope"] = pop.Rope(case["rot"], interleaved=case["interleaved"], scaling=case["scaling"], factor=case["factor"])
    return st


# ------------------------------------------------------------------------------------------------------- plain forms

def _rms(x):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)


def _plain_norm(h, u, post, gate, gain, h_scale, u_scale):
    """h' and f in fp32."""
    b = u.float()
    if post is not None:
        b = _rms(b) * post.float()
    if gate is not None:
        b = b * gate.float()
    h = h.float() * h_scale + b * u_scale
    return h, _rms(h) * gain.float()


def _plain_rows(x):
    """fp32 [T, K] -> the values that its e4m3 codes stand for (a scale for every 128 of a row), fp32 [T, K]."""
    T, K = x.shape
    pad = -K % BLOCK
    b = torch.cat([x, torch.zeros(T, pad, device=x.device)], 1).view(T, -1, BLOCK) if pad else x.view(T, -1, BLOCK)
    fine = torch.isfinite(b)
    s = (torch.where(fine, b.abs(), torch.zeros_like(b)).amax(-1, keepdim=True) * (1.0 / E4M3_MAX)).clamp(min=2.0 ** -126)
    c = (b * (1.0 / s)).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).float()
    return torch.where(fine, c * s, torch.full_like(c, math.nan)).view(T, -1)[:, :K]


def _plain_weights(codes, scales):
    N, K = codes.shape
    s = scales.repeat_interleave(BLOCK, 0)[:N].repeat_interleave(BLOCK, 1)[:, :K]
    return codes.float() * s


def _frequencies(case):
    """Angle per position of every pair (64 bits) and the factor on cosines and sines."""
    r, scaling, factor, base, start = case["rot"], case["scaling"], case["factor"], 10000.0, 4096
    i = torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / r
    if scaling == "ntk":
        base = base * factor ** (r / (r - 2))
    f = base ** -i
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "yarn":                       # pairs that turn often keep their angle, those that turn less than once are stretched
        lo, hi = (r * math.log(start / (t * 2 * math.pi)) / (2 * math.log(base)) for t in (32.0, 1.0))
        lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), r - 1)
        keep = 1 - ((torch.arange(r // 2, device=DEV, dtype=torch.float64) - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep, 0.1 * math.log(factor) + 1.0
    if scaling == "bands":                      # by the turns within the original context: under 1 stretched, over 4 kept
        keep = ((start * f / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep, 1.0
    return f, 1.0


def _plain_rotate(x, cos, sin, rot, interleaved):
    """x [T, heads, D] -> fp32, the first `rot` of every head turned."""
    x = x.float()
    y, rest = x[..., :rot], x[..., rot:]
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :rot // 2], y[..., rot // 2:])
    c, s = cos[:, None], sin[:, None]
    a, b = a * c - b * s, b * c + a * s
    y = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([y, rest], -1)


def _plain_stored(x):
    """fp32 [..., D] -> the values that the 4-bit cache holds for it: groups of 64, fp16 scale and zero point."""
    g = x.unflatten(-1, (-1, 64)).clamp(-65504.0, 65504.0)
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    s, z = ((hi - lo) * (1.0 / 15.0)).half().float(), lo.half().float()
    inv = torch.where(s > 0, 1.0 / s, torch.zeros_like(s))
    c = torch.round((g - z) * inv).clamp(0.0, 15.0)
    return (c.double() * s.double() + z.double()).float().flatten(-2)


def _plain_rope(st):
    case = st["case"]
    f, m = _frequencies(case)
    turns = torch.frac(st["pos"].double()[:, None] * (f / (2 * math.pi)))
    cos, sin = (torch.cos(turns * (2 * math.pi)) * m).float(), (torch.sin(turns * (2 * math.pi)) * m).float()
    q = _plain_rotate(st["q"], cos, sin, case["rot"], case["interleaved"])
    k = _plain_rotate(st["k"], cos, sin, case["rot"], case["interleaved"])
    dt = st["q"].dtype
    if not case["cache"]:
        return dict(q=q.to(dt), k=k.to(dt))
    return dict(q=q.to(dt), k=_plain_stored(k).to(dt), v=_plain_stored(st["v"].float()).to(dt))


def run(st):
    case = st["case"]
    if own:
        from paper_2602_06822_b200 import pop
        if case["op"] == "norm":
            h_scale, u_scale = _scales(case)
            return pop.block_norm(st["h"], st["u"], post_norm=case["post"], post_gain=st["post"], gate=st["gate"], h_scale=h_scale, u_scale=u_scale,
                                  gain=st["gain"], eps=EPS)
        if case["op"] == "linear":
            w = pop.Fp8Weights(st["codes"], st["scales"])
            if not case["norm"]:
                return pop.fp8_linear(st["x"], w)
            h, f = pop.block_norm(st["x"], st["u"], gain=st["gain"], eps=EPS, fp8=True)
            return h, pop.fp8_linear(f, w, dtype=h.dtype)
        if not case["cache"]:
            q, k = pop.rope(st["rope"], st["pos"], st["q"], st["k"])
            return dict(q=q, k=k)
        q = pop.kv_append_rope(st["pages"], st["rope"], st["pos"], st["q"], st["k"], st["v"], st["slots"])
        k, v = pop.kv_read(st["pages"], st["slots"], st["k"].dtype)
        return dict(q=q, k=k, v=v)
    if case["op"] == "norm":
        dt = st["h"].dtype
        h, f = _plain_norm(st["h"], st["u"], st["post"], st["gate"], st["gain"], *_scales(case))
        return h.to(dt), f.to(dt)
    if case["op"] == "linear":
        dt = st["x"].dtype
        w = _plain_weights(st["codes"], st["scales"]).t()
        if not case["norm"]:
            return (_plain_rows(st["x"].float()) @ w).to(dt)
        h, f = _plain_norm(st["x"], st["u"], None, None, st["gain"], 1.0, 1.0)
        return h.to(dt), (_plain_rows(f) @ w).to(dt)
    return _plain_rope(st)


# ------------------------------------------------------------------------------------------------------------ work

def work(case):
    e, T = 2 if case["dtype"] == "bf16" else 4, case["tokens"]
    if case["op"] == "norm":
        d = case["d"]
        small = d * (1 + case["post"] + (case["gate"] == "channel"))
        return dict(bytes=(T * d * (4 + (case["gate"] == "token")) + small) * e, flops=12.0 * T * d)
    if case["op"] == "linear":
        N, K = case["n"], case["k"]
        blocks = -(-N // BLOCK) * -(-K // BLOCK)
        return dict(bytes=N * K + 4 * blocks + (T * K * (3 if case["norm"] else 1) + T * N) * e, flops=2.0 * T * N * K)
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    if not case["cache"]:
        return dict(bytes=2 * T * (H + Hk) * D * e + 4 * T, flops=3.0 * T * (H + Hk) * case["rot"])
    tile = D // 64 * (2 * 512 + 16 * 8)
    return dict(bytes=T * (2 * H + 4 * Hk) * D * e + 2 * T * Hk * tile / 16 + 12 * T, flops=3.0 * T * (H + Hk) * case["rot"])


# ----------------------------------------------------------------------------------------------------------- exact

def _norm64(h, u, post, gate, gain, h_scale, u_scale):
    block = u.double()
    if post is not None:
        block = block * ((block ** 2).sum(1, keepdim=True) / block.shape[1] + EPS).rsqrt() * post.double()[None]
    if gate is not None:
        block = block * gate.double()
    new = h_scale * h.double() + u_scale * block
    return new, new * ((new ** 2).sum(1, keepdim=True) / new.shape[1] + EPS).rsqrt() * gain.double()[None]


def _e4m3_64(x, s):
    """x (64 bits) as the multiple of s that its code says, by e4m3's definition: 3 bits behind the leading one, steps of 2^-9 at
    least, 448 at most, ties to even.  x / s is decided as the product with the reciprocal, both in binary32."""
    r = (x.float() * (1.0 / s.float())).double()
    step = torch.exp2((torch.floor(torch.log2(r.abs().clamp(min=2.0 ** -6))) - 3))
    return (torch.round(r / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _product64(x, codes, scales):
    """sum over blocks of scale * scale * (sum of products of codes), 64 bits."""
    out = torch.zeros(x.shape[0], codes.shape[0], dtype=torch.float64, device=x.device)
    for b, k in enumerate(range(0, x.shape[1], BLOCK)):
        part = x[:, k:k + BLOCK].double()
        s = torch.clamp((part.abs().max(1, keepdim=True).values.float() * float(np.float32(1.0 / E4M3_MAX))), min=2.0 ** -126).double()
        of_row = scales[torch.arange(codes.shape[0], device=x.device) // BLOCK, b].double()
        out += (_e4m3_64(part, s) * s) @ (codes[:, k:k + BLOCK].double() * of_row[:, None]).T
    return out


def _turned64(x, angle, m, rot, interleaved):
    """Rotation by `angle` [T, rot / 2]: cosine and sine (times m) rounded to binary32, then every product and sum, as the cache's
    quantiser sees them."""
    c, s = ((fn(angle) * m).float().double()[:, None, :] for fn in (torch.cos, torch.sin))
    y = x.double().clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., first].double(), x[..., second].double()
    r32 = lambda t: t.float().double()                                       # noqa: E731
    y[..., first] = r32(r32(a * c) - r32(b * s))
    y[..., second] = r32(r32(b * c) + r32(a * s))
    return y


def _stored64(x):
    """What the 4-bit cache holds for x [T, H, D] (64 bits), by its format's definition."""
    out = torch.empty_like(x)
    for a in range(0, x.shape[2], 64):
        y = x[:, :, a:a + 64]
        least, most = y.min(2, keepdim=True).values, y.max(2, keepdim=True).values
        scale = ((most - least).float().double() * float(np.float32(1.0 / 15.0))).float().half().double()
        zero = least.half().double()
        per = torch.where(scale == 0, torch.zeros_like(scale), (1.0 / scale).float().double())
        code = ((y - zero).float().double() * per).float().double().round().clamp(0, 15)
        out[:, :, a:a + 64] = zero + scale * code
    return out


def _angles64(case, pos):
    """[T, rot / 2] angles, whole turns taken off, from the frequencies' definition written pair by pair."""
    r, factor, start, out = case["rot"], case["factor"], 4096.0, []
    for i in range(r // 2):
        base = 10000.0 * (factor ** (r / (r - 2.0)) if case["scaling"] == "ntk" else 1.0)
        f = 1.0 / base ** (2.0 * i / r)
        if case["scaling"] == "linear":
            f /= factor
        elif case["scaling"] == "yarn":
            place = [r * math.log(start / (2 * math.pi * t)) / (2 * math.log(base)) for t in (32.0, 1.0)]
            low, high = max(0, math.floor(place[0])), min(r - 1, math.ceil(place[1]))
            slope = min(1.0, max(0.0, (i - low) / max(high - low, 1e-3)))
            f = f * (1 - slope) + f / factor * slope
        elif case["scaling"] == "bands":
            slope = min(1.0, max(0.0, (start * f / (2 * math.pi) - 1.0) / 3.0))
            f = f / factor * (1 - slope) + f * slope
        turns = pos.double() * (f / (2 * math.pi))
        out.append((turns - turns.floor()) * (2 * math.pi))
    return torch.stack(out, 1), 0.1 * math.log(factor) + 1.0 if case["scaling"] == "yarn" else 1.0


def exact(case, seed):
    if case["op"] == "norm":
        return _norm64(*_norm_inputs(case, seed), *_scales(case))
    if case["op"] == "linear":
        x, u, gain, codes, scales = _linear_inputs(case, seed)
        if not case["norm"]:
            return _product64(x, codes, scales)
        h, f = _norm64(x, u, None, None, gain, 1.0, 1.0)
        return h, _product64(f, codes, scales)
    q, k, v, pos = _rope_inputs(case, seed)
    angle, m = _angles64(case, pos)
    q, k = (_turned64(t, angle, m, case["rot"], case["interleaved"]) for t in (q, k))
    if not case["cache"]:
        return dict(q=q, k=k)
    return dict(q=q, k=_stored64(k), v=_stored64(v.double()))
