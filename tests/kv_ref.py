"""The paged key/value cache and its attention in 64 bits, on the CPU: a token,
a row and a head at a time from the definitions, without the library's code."""

import numpy as np
import torch

E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6])


def positions(offsets, lens, rows):
    """(sequence, position) of every row; sequence -1: padding."""
    seq, pos = np.full(rows, -1, np.int64), np.zeros(rows, np.int64)
    for s in range(len(lens)):
        n = offsets[s + 1] - offsets[s]
        seq[offsets[s]:offsets[s + 1]] = s
        pos[offsets[s]:offsets[s + 1]] = lens[s] - n + np.arange(n)
    return seq, pos


def rotate32(x, cos, sin):
    """x [rows, heads, D], cos, sin [rows, D / 2], all fp32: every product and sum rounded to fp32."""
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h], x[..., h:], cos[:, None], sin[:, None]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def mx_quantize(x, rule="floor"):
    """fp32 [..., D] -> (codes [..., D], scale codes [..., D / 32]) in 64 bits, value by value of the grid."""
    b = x.astype(np.float64).reshape(x.shape[:-1] + (-1, 32))
    peak = np.abs(b).max(-1)
    safe = np.where(peak > 0, peak, 1.0)
    m, e = np.frexp(safe)                       # peak = m 2^e, m in [0.5, 1)
    ex = e - 1 - 2 if rule == "floor" else np.where(m > 0.75, e - 2, e - 3)   # ceil(log2(peak / 6)), 6 = 0.75 * 8
    ex = np.where(peak > 0, np.maximum(ex, -127), -127)
    a = np.abs(b) / np.exp2(ex.astype(np.float64))[..., None]
    grid = E2M1[:8]
    mid = (grid[1:] + grid[:-1]) / 2
    code = np.zeros(a.shape, np.uint8)
    for i, t in enumerate(mid):                 # a tie goes to the even code
        code += (a >= t) if i % 2 else (a > t)
    code |= np.where(np.signbit(b), 8, 0).astype(np.uint8)
    return code.reshape(x.shape), (ex + 127).astype(np.uint8)


def mx_values(codes, scales):
    v = E2M1[codes].reshape(codes.shape[:-1] + (-1, 32)) * np.exp2(scales.astype(np.float64) - 127)[..., None]
    return v.reshape(codes.shape)


def unpack(packed):
    return np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[:-1] + (-1,))


def pool_values(cache):
    """(k, v) [pages, heads, page_size, D] of a KVCache, in 64 bits."""
    if cache.fmt == "bf16":
        return tuple(t.cpu().double().numpy() for t in (cache.k, cache.v))
    return tuple(mx_values(unpack(t.cpu().numpy()), e.cpu().numpy())
                 for t, e in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))


def attention(q, kpool, vpool, offsets, lens, table, scale, window=0, sinks=0, prefix_table=None, prefix_len=0):
    """q [rows, heads, D] float64.  Returns (o [rows, heads, D], lse [rows, heads], sum w|v| like o, the largest
    |q|.|k| a score sums, [rows, heads]).  Rows of no sequence: NaN."""
    rows, hq, D = q.shape
    pages, hkv, ps, _ = kpool.shape
    g = hq // hkv
    o, mag = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, size = np.full((rows, hq), np.nan), np.zeros((rows, hq))
    seq, pos = positions(offsets, lens, rows)
    for i in range(rows):
        if seq[i] < 0:
            continue
        p = pos[i]
        t = np.arange(max(p + 1, 0))
        if window:
            t = t[(p - t < window) | (t < sinks)]
        page = np.array([prefix_table[x // ps] if x < prefix_len else table[seq[i]][x // ps] for x in t], np.int64)
        ok = (page >= 0) & (page < pages)
        t, page = t[ok], page[ok]
        o[i], mag[i], lse[i] = 0.0, 0.0, -np.inf
        if len(t) == 0:
            continue
        for h in range(hkv):
            k, v = kpool[page, h, t % ps], vpool[page, h, t % ps]
            z = q[i, h * g:(h + 1) * g] @ k.T * scale
            top = z.max(-1, keepdims=True)
            w = np.exp(z - top)
            l = w.sum(-1, keepdims=True)
            sl = slice(h * g, (h + 1) * g)
            o[i, sl], mag[i, sl] = w @ v / l, w @ np.abs(v) / l
            lse[i, sl] = (top + np.log(l))[:, 0]
            size[i, sl] = (np.abs(q[i, sl]) @ np.abs(k).T).max(-1)
    return o, lse, mag, size


def tolerance(o, mag, size, D, scale, n, vmax):
    """How far an output may be from `o`.  Rounding the output to bf16 costs half a step, 2^-8 of the value; rounding
    the weights to bf16 at most 2^-8 of sum w|v| (their sum l is not rounded).  A score sums D products in fp32
    (2^-24 of |q|.|k| each) and is scaled and shifted (2^-23 of it twice): an error d of a score moves its weight and
    the sum by a factor e^d each.  exp2 and the fp32 sums over n tokens cost n 2^-24 + 2^-21 of sum w|v|.  A weight
    below 2^-126 of the largest has no normal fp32 or bf16 number and may be lost, with its product of at most vmax."""
    d = size[..., None] * scale * (D + 4) * 2.0 ** -24
    return 2.0 ** -8 * np.abs(o) + mag * ((1 + 2.0 ** -8) * 2.0 ** -8 + 2 * np.expm1(d) + n * 2.0 ** -23 + 2.0 ** -20) + \
        n * vmax * 2.0 ** -125


def lse_tolerance(lse, size, D, scale, n):
    """The scores' error, n + 4 roundings of the sum, and the logarithm's in base 2."""
    return size * scale * (D + 4) * 2.0 ** -24 + (n + 4) * 2.0 ** -24 + 2.0 ** -20 + np.abs(lse) * 2.0 ** -21


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)
