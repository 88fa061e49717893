"""Inputs of the attention under which a single token of a long sequence shows in
the result, with the result that they must give.  (Under random inputs one token
of thousands weighs less than the output's rounding.)"""

import numpy as np


def counting_values(n, heads, D, rng):
    """[n, heads, D]: every token has a single 1, in a column that it shares with about n / D others.  With queries of
    zero all weights are the same, and column d of the output is the number of its tokens that are visible over the
    number of all that are."""
    v = np.zeros((n, heads, D), np.float32)
    for h in range(heads):
        v[np.arange(n), h, rng.permutation(n) % D] = 1.0
    return v


def visible(p, length, window=0, sinks=0):
    """bool [length]: the tokens that a row at position p sees."""
    t = np.arange(length)
    return (t <= p) & ((p - t < window) | (t < sinks) if window else True)


def counted(v, p, window=0, sinks=0):
    """The output [heads, D] in 64 bits of a row at position p over values v [n, heads, D] with queries of zero, and its
    lse."""
    see = visible(p, len(v), window, sinks)
    n = int(see.sum())
    return v[see].sum(0, dtype=np.float64) / max(n, 1), np.log(n) if n else -np.inf


def count_tolerance(o):
    """Scores of zero are exact, and so are weights of 1, their sums (whole numbers below 2^24) and the sums of ones and
    zeros; the reciprocal and the product round to fp32 (2^-24 each), the output to bf16 (2^-8)."""
    return (2.0 ** -8 + 2.0 ** -22) * o


def count_lse_tolerance(lse):
    """log2 of an exact sum (an ulp of its result), times ln 2 rounded to fp32, rounded once more."""
    return np.abs(lse) * 2.0 ** -21


PEAK = 6.0


def pick_targets(positions, heads, q_heads, rng, low=0, taken=None):
    """A token for every row (at `positions`) and query head, at most its position and at least `low`: no token twice for a
    key/value head.  First, last and tokens beside multiples of 16 come before others.  int [rows, q_heads], -1: none
    was left.  taken: sets a head, extended."""
    group = q_heads // heads
    taken = taken if taken is not None else [set() for _ in range(heads)]
    out = np.full((len(positions), q_heads), -1, np.int64)
    for i, p in enumerate(positions):
        edges = np.array([t for t in range(low, p + 1) if t % 16 in (0, 15) or t == p])
        for h in range(q_heads):
            left = [t for t in rng.permutation(edges)[:40] if t not in taken[h // group]] if len(edges) else []
            left += [t for t in rng.integers(low, p + 1, 40) if t not in taken[h // group]] if p >= low else []
            if left:
                out[i, h] = left[0]
                taken[h // group].add(int(left[0]))
    return out


def aim(k, q, targets):
    """Into keys k [n, heads, D] at every row's and head's target a multiple of its query q [rows, q_heads, D]: the
    target then takes all but a negligible part of the row's weight."""
    group = q.shape[1] // k.shape[1]
    for i, h in np.argwhere(targets >= 0):
        k[targets[i, h], h // group] = PEAK * q[i, h]
