"""Microscaled 4-bit numbers, their product and attention over a cache of them in plain 64-bit numpy, one element at a time where that is
affordable: what the GPU tests compare with.  Written from the format's definition in include/sfs.h."""
import math

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])
MATRIX, CACHE = (0, 254), (65, 192)


def nearest_code(y):
    """Code of the nearest magnitude to |y|, ties to the even code."""
    d = np.abs(np.abs(y)[..., None] - MAGNITUDES)
    best = d.min(-1, keepdims=True)
    tied = d == best
    even = tied & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), tied.argmax(-1))
    return code + 8 * (np.signbit(y) & ~np.isnan(y))


def quantize(x, lo_hi):
    """x [..., n] -> (codes 0..15 [..., 32 blocks], scales [..., blocks])."""
    lo, hi = lo_hi
    x = np.asarray(x, dtype=np.float64)
    pad = -x.shape[-1] % 32
    b = np.concatenate([x, np.zeros(x.shape[:-1] + (pad,))], -1).reshape(x.shape[:-1] + (-1, 32))
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    a = np.abs(b).max(-1)
    c = np.full(a.shape, lo, dtype=np.int64)
    e = np.frexp(a)[1] - 1                                  # floor(log2 a): frexp's mantissa lies in [0.5, 1)
    c = np.where(a > 0, np.clip(e - 2 + 127, lo, hi), c)
    codes = nearest_code(np.ldexp(b, (127 - c)[..., None]))
    codes = np.where(bad[..., None], 0, codes).reshape(x.shape[:-1] + (-1,))
    return codes.astype(np.uint8), np.where(bad, 255, c).astype(np.uint8)


def values(codes, scales, nan_above=254):
    c = scales.astype(np.int64)
    f = np.where(c > nan_above, np.nan, np.ldexp(1.0, np.minimum(c, 254) - 127))
    return VALUES[codes] * np.repeat(f, 32, -1)


def pack(codes):
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(packed):
    out = np.empty(packed.shape[:-1] + (2 * packed.shape[-1],), dtype=np.uint8)
    out[..., 0::2], out[..., 1::2] = packed & 15, packed >> 4
    return out


def scale_places(rows, blocks):
    r, b = np.arange(rows)[:, None], np.arange(blocks)[None]
    return ((r // 128) * ((blocks + 3) // 4) + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4


def tile_scales(scales):
    rows, blocks = scales.shape
    out = np.zeros((rows + 127) // 128 * ((blocks + 3) // 4) * 512, dtype=np.uint8)
    out[scale_places(rows, blocks)] = scales
    return out


def seen(length, p, left, right, sinks):
    """Truth values over the keys: what a row at position p sees."""
    j = np.arange(length)
    s = np.ones(length, dtype=bool)
    if right >= 0:
        s &= j <= p + right
    if left >= 0:
        s &= (j >= p - left) | (j < sinks)
    return s


def attention(q, k, v, mask):
    """One head: q [n, d], k and v [m, d], mask [n, m] -> (out, bound): the rows' outputs, and how far rounded probabilities and 32-bit
    sums can be from them before the output itself is rounded.

    bound per element, with A = sum_j p_j |v_j|: probabilities rounded to bf16, 2^-8 A; a score is a sum of d products in 32 bits, off by
    at most d 2^-24 sum_d |q_d k_d| / sqrt(d) in any order, which moves a probability by that factor in numerator and denominator; the
    exponential (2^-21), the denominator and the sum over m keys in 32 bits (m 2^-24 each) together 2^-21 + 2 m 2^-24.  A probability
    below 2^-126 of a reference that may lag the row's maximum by 2^8 is no normal 32-bit number and counts as 0: 2^-118 |v_j| each."""
    n, d = q.shape
    if len(k) and all(np.isfinite(x).all() for x in (q, k, v)):
        s = np.where(mask, q @ k.T / math.sqrt(d), -np.inf)
        some = mask.any(1)
        w = np.zeros_like(s)
        w[some] = np.exp(s[some] - s[some].max(1, keepdims=True, initial=-np.inf))
        w[some] /= w[some].sum(1, keepdims=True)
        off = d * 2.0 ** -24 * np.where(mask, np.abs(q) @ np.abs(k).T, 0.0).max(1, initial=0.0, keepdims=True) / math.sqrt(d)
        a, seen_values = w @ np.abs(v), mask.astype(float) @ np.abs(v)
        return w @ v, 2.0 ** -118 * seen_values + a * (2.0 ** -8 + 2 * np.expm1(np.minimum(off, 1.0)) + 2.0 ** -21 + 2 * mask.sum(1, keepdims=True) * 2.0 ** -24)
    out, bound = np.zeros((n, d)), np.zeros((n, d))
    for i in range(n):                                      # row by row where something is not finite: what a row does not see must not reach it
        at = np.flatnonzero(mask[i])
        if at.size == 0:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            s = k[at] @ q[i] / math.sqrt(d)
            w = np.exp(s - s.max())
            w = w / w.sum()
            out[i] = w @ v[at]
            a = w @ np.abs(v[at])
            off = d * 2.0 ** -24 * (np.abs(k[at]) @ np.abs(q[i])).max() / math.sqrt(d)
            bound[i] = 2.0 ** -118 * np.abs(v[at]).sum(0) + a * (2.0 ** -8 + 2 * math.expm1(min(off, 1.0)) + 2.0 ** -21 + 2 * at.size * 2.0 ** -24)
    return out, bound
