"""Oracle of what a decoder layer does around its attention (pop_block_norm, pop_fp8_quantize, pop_fp8_linear, pop_rope): numpy, 64 bits, test
infrastructure only.  Where the public description fixes the arithmetic (scales and codes, the rotation's roundings) it is done in that
arithmetic, everything else in 64 bits."""
import math

import numpy as np

BLOCK = 128
F32 = np.float32


# ------------------------------------------------------------------------------------------------------------------ norms

def block_norm(h, u=None, post_norm=False, post_gain=None, gate=None, h_scale=1.0, u_scale=1.0, gain=None, eps=1e-5):
    """(h', f, b): the new stream, what the next block gets, and the block's part of h' (u_scale gate b)."""
    rms = lambda x: x / np.sqrt((x * x).mean(1, keepdims=True) + eps)        # noqa: E731
    h = np.asarray(h, dtype=np.float64) * h_scale
    b = np.zeros_like(h)
    if u is not None:
        b = np.asarray(u, dtype=np.float64)
        if post_norm:
            b = rms(b) * (1.0 if post_gain is None else np.asarray(post_gain, dtype=np.float64))
        if gate is not None:
            b = b * np.asarray(gate, dtype=np.float64)
        b = b * u_scale
    new = h + b
    return new, rms(new) * (1.0 if gain is None else np.asarray(gain, dtype=np.float64)), b


# ------------------------------------------------------------------------------------------------------------------- fp8

def _code_table():
    """The 256 values of e4m3: bias 7, 3 bits behind the leading one, no infinities, all ones NaN."""
    out = np.zeros(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = math.nan if c & 127 == 127 else -v if c & 128 else v
    return out


CODES = _code_table()
_POSITIVE = CODES[:127]                          # ascending, 0 .. 448


def code_of(x):
    """The code nearest to each of x (ties to the even code); beyond 448 as 448, what is not finite NaN."""
    a = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), 448.0)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POSITIVE[lo], _POSITIVE[hi] - a
    c = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    c = c + 128 * np.signbit(x)
    return np.where(np.isfinite(x), c, 127).astype(np.uint8)


def quantise(x, block_rows):
    """codes uint8 [rows, K] and scales (float32; [ceil(K / 128), rows], or [ceil(rows / 128), ceil(K / 128)] for weights)."""
    x = np.asarray(x, dtype=F32)
    rows, K = x.shape
    R, KB = -(-rows // block_rows), -(-K // BLOCK)
    codes, scales = np.zeros((rows, K), dtype=np.uint8), np.zeros((R, KB), dtype=F32)
    for r in range(R):
        for b in range(KB):
            at = np.s_[r * block_rows:(r + 1) * block_rows, b * BLOCK:(b + 1) * BLOCK]
            v = x[at]
            top = np.max(np.abs(np.where(np.isfinite(v), v, F32(0))), initial=F32(0))
            s = max(F32(top * F32(1 / 448)), F32(2.0 ** -126))
            scales[r, b] = s
            with np.errstate(invalid="ignore"):
                codes[at] = code_of((v * (F32(1) / s)).astype(np.float64))
    return codes, (np.ascontiguousarray(scales.T) if block_rows == 1 else scales)


def values(codes, scales, block_rows):
    """What the codes stand for, 64 bits."""
    s = np.asarray(scales, dtype=np.float64)
    s = s.T if block_rows == 1 else np.repeat(s, BLOCK, 0)[:codes.shape[0]]
    return CODES[codes] * np.repeat(s, BLOCK, 1)[:, :codes.shape[1]]


# ------------------------------------------------------------------------------------------------------------------ rope

def rope_frequencies(rot, base=10000.0, scaling="none", factor=1.0, original=4096.0, fast=None, slow=1.0):
    """(angles per position [rot / 2] in 64 bits, magnitude)."""
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    w = np.array([base ** (-2.0 * i / rot) for i in range(rot // 2)])
    if scaling == "linear":
        return w / factor, 1.0
    if scaling == "yarn":
        at = lambda t: rot * math.log(original / (t * 2 * math.pi)) / (2 * math.log(base))      # noqa: E731
        lo, hi = max(math.floor(at(32.0 if fast is None else fast)), 0), min(math.ceil(at(slow)), rot - 1)
        keep = 1 - np.clip((np.arange(rot // 2) - lo) / max(hi - lo, 1e-3), 0, 1)
        return w * keep + w / factor * (1 - keep), 0.1 * math.log(factor) + 1
    if scaling == "bands":
        keep = np.clip((original * w / (2 * math.pi) - slow) / ((4.0 if fast is None else fast) - slow), 0, 1)
        return w * keep + w / factor * (1 - keep), 1.0
    return w, 1.0


def cos_sin(freq, magnitude, positions):
    """float32 [T, pairs] each, from frequencies in 2^-64 turns: whole turns are dropped in integers."""
    part = np.array([[int(p) * int(f) % 2 ** 64 for f in freq] for p in positions], dtype=np.uint64).view(np.int64).reshape(len(positions), len(freq))
    angle = part.astype(np.longdouble) * (np.longdouble(2.0) ** -63 * np.longdouble("3.14159265358979323846264338327950288"))
    m = np.longdouble(magnitude)
    return (np.cos(angle) * m).astype(np.float64).astype(F32), (np.sin(angle) * m).astype(np.float64).astype(F32)


def rotate(x, cos, sin, interleaved, inverse=False):
    """x [T, heads, D] (values of fp32) -> float32, every product and sum rounded."""
    x = np.asarray(x, dtype=F32)
    pairs = cos.shape[1]
    c, s = cos[:, None], (-sin if inverse else sin)[:, None]
    ia, ib = (np.arange(pairs) * 2, np.arange(pairs) * 2 + 1) if interleaved else (np.arange(pairs), np.arange(pairs) + pairs)
    y = x.copy()
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y
