"""The 4-bit cache by its definition, in float64 on the CPU: what a group of 32 values is rounded to, how the bytes lie, and
attention over the values that the bytes stand for."""
import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def f64(bits):
    """bf16 patterns (uint16) -> float64."""
    with np.errstate(invalid="ignore"):
        return (np.ascontiguousarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def to_bf16_bits(x):
    """float64 that bf16 holds exactly -> patterns."""
    with np.errstate(over="ignore"):
        f = np.asarray(x, np.float64).astype(np.float32)
    return (f.view(np.uint32) >> 16).astype(np.uint16)


def quantise(x):
    """x [..., 32 n] float64 -> codes 0..15 [..., n, 32], scale bytes [..., n]."""
    x = x.reshape(*x.shape[:-1], -1, 32)
    finite = np.isfinite(x).all(-1)
    y = np.where(finite[..., None], x, 0.0)
    amax = np.abs(y).max(-1)
    b = 2 + np.searchsorted(7.0 * 2.0 ** (np.arange(2, 252) - 127.0), amax, side="right")   # the smallest scale of which 7 are more than amax
    r = np.abs(y) / (2.0 ** (b - 127.0))[..., None]
    d = np.abs(r[..., None] - LEVELS)
    near = d.min(-1, keepdims=True)
    tie = d == near
    even = tie & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), tie.argmax(-1))
    code = code + 8 * np.signbit(y)
    return code.astype(np.uint8), np.where(finite, b, 255).astype(np.uint8)


def values(codes, scales):
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127.0))
    v = np.where(codes >= 8, -1.0, 1.0) * LEVELS[codes & 7]
    v = v * s[..., None]
    return v.reshape(*v.shape[:-2], -1)


def rounded(x):
    return values(*quantise(x))


def places(hd, t):
    """Byte offsets, within a (block, head), of token slot t: K codes [g, 16], V codes [g, 16], K scales [g], V scales [g]."""
    G = hd // 32
    g, j = np.arange(G)[:, None], np.arange(16)
    kc = (g * 16 + t) * 16 + j
    vc = 8 * hd + (((t // 4) * 16 + j) * G + g) * 4 + t % 4
    ks = 16 * hd + np.arange(G) * 16 + t
    vs = 16 * hd + hd // 2 + ((t // 4) * G + np.arange(G)) * 4 + t % 4
    return kc, vc, ks, vs


def put(pool, hd, blk, t, k, v):
    """Quantises one token's k, v [heads, hd] float64 into pool [n_blocks, heads, 17 hd] at (blk, t)."""
    kc, vc, ks, vs = places(hd, t)
    for where_c, where_s, x in ((kc, ks, k), (vc, vs, v)):
        c, s = quantise(x)
        pool[blk][:, where_c] = c[..., 0::2] | (c[..., 1::2] << 4)
        pool[blk][:, where_s] = s


def get(pool, hd, blk, t):
    kc, vc, ks, vs = places(hd, t)
    out = []
    for where_c, where_s in ((kc, ks), (vc, vs)):
        byte = pool[blk][:, where_c]
        codes = np.stack((byte & 15, byte >> 4), -1).reshape(*byte.shape[:-1], 32)
        out.append(values(codes, pool[blk][:, where_s]))
    return out


def gather(pool, hd, table, n):
    """Keys and values [n, heads, hd] of a request's first n tokens."""
    both = [get(pool, hd, int(table[t // 16]), t % 16) for t in range(n)]
    heads = pool.shape[1]
    return np.array([k for k, _ in both]).reshape(n, heads, hd), np.array([v for _, v in both]).reshape(n, heads, hd)


def attention(q, k, v, first):
    """q [rows, Hq, hd] at positions first.. over k, v [n, Hkv, hd], causal.  Returns the output and a bound of what rounding may
    do to it, element by element (float64):

    every weight is rounded to bf16 (2^-8 of itself), once in the numerator and once in the sum, which is taken of the rounded or
    of the unrounded ones; its score is off by delta and so itself by as much relatively, again in both; delta is what the query's
    terms leave of it, at most 2^-13 of the largest of the 32 dims for each (2^-13.9, and float32's rounding of the product with
    the scale), and 2^-14 of sum|q k| for the sums in the matrix unit and the maximum that they start from (2^-15.7 at most was
    measured with products of more bits); the exponential and the sums in float32 are within 2^-16; and the result is rounded to
    bf16 (2^-8 of itself, once more for the error in front of it)."""
    rows, Hq, hd = q.shape
    G = Hq // k.shape[1]
    out, bound = np.zeros((rows, Hq, hd)), np.zeros((rows, Hq, hd))
    for r in range(rows):
        n = first + r + 1
        if n <= 0:
            continue
        for h in range(Hq):
            kk, vv = k[:n, h // G], v[:n, h // G]
            s = kk @ q[r, h] / math.sqrt(hd)
            top = np.repeat(np.abs(q[r, h]).reshape(-1, 32).max(1), 32)
            delta = float(np.max(np.abs(kk) @ (2.0 ** -14 * np.abs(q[r, h]) + 2.0 ** -13 * top))) / math.sqrt(hd)
            p = np.exp(s - s.max())
            p /= p.sum()
            out[r, h] = p @ vv
            e = (p @ np.abs(vv)) * (2.0 ** -8 + 2.0 * delta + 2.0 ** -16) + 2.0 ** -8 * np.abs(p @ vv)
            bound[r, h] = e + 2.0 ** -8 * (np.abs(out[r, h]) + e)
    return out, bound
