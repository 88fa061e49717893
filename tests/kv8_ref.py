"""The 8-bit key/value cache in 64 bits, on the CPU: codes, scales and the append, block by block from the definition."""

import numpy as np
import torch

import kv_ref as R

BLOCK, TOP, LEAST = 16, 448.0, -117

_C = np.arange(256)
_E, _M = _C >> 3 & 15, _C & 7
#: the value of every E4M3 code
VALUES = np.where(_E == 0, _M / 8 * 2.0 ** -6, (1 + _M / 8) * np.exp2(_E - 7.0)) * np.where(_C < 128, 1, -1)
VALUES[[0x7F, 0xFF]] = np.nan


def encode(x):
    """64-bit values -> the nearest codes, ties to the even one, saturating; what is not finite: NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.where(np.isfinite(x), np.abs(x), 0), TOP)
    grid = VALUES[:0x7F]
    hi = np.searchsorted(grid, a)                        # grid[hi - 1] < a <= grid[hi]
    lo = np.maximum(hi - 1, 0)
    up = (a - grid[lo] > grid[hi] - a) | ((a - grid[lo] == grid[hi] - a) & (hi % 2 == 0))
    code = np.where(up, hi, lo).astype(np.uint8) | np.where(np.signbit(x), 0x80, 0).astype(np.uint8)
    return np.where(np.isfinite(x), code, 0x7F).astype(np.uint8)


def exponent(peak, rule="floor"):
    """Exponent of the scale of a block whose largest finite magnitude is `peak`."""
    if peak == 0:
        return LEAST
    m, e = np.frexp(np.float64(peak))                    # peak = m 2^e; 448 = 0.875 * 2^9
    return max(int(e) - 9 + (1 if rule == "ceil" and m > 0.875 else 0), LEAST)


def quantize(x, rule="floor"):
    """[pages, heads, page, D] -> (codes, scale codes [pages, heads, page / 16])."""
    b = x.astype(np.float64).reshape(x.shape[:2] + (-1, BLOCK, x.shape[3]))
    peak = np.abs(b).max((-1, -2))
    e = np.vectorize(lambda p: exponent(p, rule), otypes=[np.int64])(peak)
    return encode(b / np.exp2(e.astype(float))[..., None, None]).reshape(x.shape), (e + 127).astype(np.uint8)


def values(codes, scales):
    """In 64 bits, like `codes`."""
    with np.errstate(over="ignore", invalid="ignore"):
        s = np.exp2(scales.astype(np.float64) - 127)
        s[scales == 0xFF] = np.nan
        v = VALUES[codes].reshape(codes.shape[:2] + (-1, BLOCK, codes.shape[3])) * s[..., None, None]
    return v.reshape(codes.shape)


def append(pools, k, v, offsets, lens, table, page, rule="floor", skip=None):
    """pools: [codes k, codes v, scales k, scales v], changed in place.  k, v: fp32 [rows, heads, D], rotated.
    skip: rows that are left out."""
    pages, heads = pools[0].shape[:2]
    for s in range(len(lens)):
        n = offsets[s + 1] - offsets[s]
        base = int(lens[s]) - int(n)
        for b in range(max(base, 0) // BLOCK, -(-max(int(lens[s]), 0) // BLOCK)):
            pos = [p for p in range(max(base, b * BLOCK), min(int(lens[s]), (b + 1) * BLOCK)) if p >= 0]
            rows = [int(offsets[s]) + p - base for p in pos]
            there = [(p, r) for p, r in zip(pos, rows) if skip is None or not skip[r]]
            pg = table[s][b * BLOCK // page] if there else -1
            if not 0 <= pg < pages:
                continue
            old = max(base - b * BLOCK, 0)
            first, at = b * BLOCK % page, b * BLOCK % page // BLOCK
            for x, codes, scales in ((k, pools[0], pools[2]), (v, pools[1], pools[3])):
                for h in range(heads):
                    new = np.array([x[r, h] for _, r in there], np.float64)
                    fine = np.abs(new[np.isfinite(new)])
                    e = exponent(fine.max(initial=0.0), rule)
                    if old:
                        before = int(scales[pg, h, at]) - 127
                        e = max(e, before)
                        part = codes[pg, h, first:first + old]
                        if e > before:
                            part[:] = encode(VALUES[part] * 2.0 ** (before - e))
                    for (p, _), y in zip(there, new):
                        codes[pg, h, p % page] = encode(y * 2.0 ** -e)
                    scales[pg, h, at] = e + 127


def pool_values(cache):
    """(k, v) [pages, heads, page_size, D] of a KVCache of any format, in 64 bits."""
    if cache.fmt != "fp8":
        return R.pool_values(cache)
    u8 = lambda t: t.cpu().view(torch.uint8).numpy()  # noqa: E731
    return tuple(values(u8(c), u8(e)) for c, e in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
