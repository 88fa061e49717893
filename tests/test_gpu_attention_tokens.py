"""Attention over long sequences with inputs under which every single token shows
in the result: which tokens are read, with which values, once each, whatever
workgroups and wavefronts share them."""

import numpy as np
import pytest
import torch

import kv_ref as R
import kv_tokens as T
from paper_2606_26587_amd import sharq as S
from test_gpu_attention import FMTS, check
from test_gpu_kv import DEV, make_batch

pytestmark = pytest.mark.gpu

HQ, HKV = 8, 2

CASES = [
    # rows, lengths, page, prefix, window, sinks
    ([1], [9000], 64, 0, 0, 0),
    ([1, 3, 2], [6000, 10, 3500], 64, 0, 0, 0),
    ([9], [5000], 64, 0, 0, 0),
    ([30, 18], [3000, 700], 16, 0, 0, 0),
    ([1] * 3, [5000, 4100, 4500], 64, 4096, 0, 0),
    ([25, 1], [2300, 2100], 32, 2048, 0, 0),
    ([8, 5, 1], [2900, 2100, 2500], 16, 1024, 0, 0),
    ([1, 1, 3], [2500, 1300, 4100], 64, 0, 1024, 4),
    ([40, 2], [3000, 1900], 128, 0, 1000, 70),
    ([2, 1], [3000, 2600], 64, 1024, 900, 130),             # the window leaves most of a prefix
    ([300], [1500], 16, 0, 0, 0),
    ([150, 1, 4, 1] + [1] * 40, [700, 3000, 2000, 1025] + [300 + 17 * i for i in range(40)], 32, 0, 0, 0),
    ([1] * 70, [900 + 31 * i for i in range(70)], 64, 0, 0, 0),
]


def pool_of(seqs, table, pages, page, prefix):
    """[pages, heads, page, D] fp32 from the sequences' [n, heads, D]; tokens of the prefix are the longest one's."""
    n, heads, D = seqs[0].shape
    pool = np.full((pages, page, heads, D), np.nan, np.float32)
    longest = int(np.argmax([len(s) for s in seqs]))
    for i, x in enumerate(seqs):
        t = np.arange(0 if i == longest else prefix, len(x))
        pool[table[i, t // page], t % page] = x[t]
    return np.ascontiguousarray(pool.transpose(0, 2, 1, 3))


def cache_of(k, v, fmt):
    """A cache of these pools; slots that hold NaN (no sequence's) get what is no number in the cache's format."""
    if fmt == "bf16":
        return S.KVCache(fmt, R.bf16(k).to(DEV), R.bf16(v).to(DEV))
    parts = []
    for x in (k, v):
        none = np.isnan(x)
        c, e = R.mx_quantize(np.where(none, 0, x).astype(np.float32))
        c[none] = 15
        e[none[..., ::32]] = 0xFF
        parts.append((torch.from_numpy(c[..., 0::2] | c[..., 1::2] << 4).to(DEV), torch.from_numpy(e).to(DEV)))
    return S.KVCache(fmt, parts[0][0], parts[1][0], parts[0][1], parts[1][1])


def batch_of(per, lens, page, prefix, seed):
    batch, offsets, lens, table, pages = make_batch(per, lens, page, seed=seed)
    own = table.copy()
    pt = None
    if prefix:
        pt = table[int(np.argmax(lens)), :prefix // page].copy()
        own[:, :prefix // page] = -7                        # not looked at
        batch.page_table.copy_(torch.from_numpy(own))
    return batch, offsets, lens, table, own, pages, pt


def call(q, cache, batch, window, sinks, pt, prefix):
    out = torch.full((batch.rows, q.shape[1]), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((batch.rows, HQ), 9.0, device=DEV)
    S.sharq_attention(q, cache, batch, window=window, sinks=sinks, out=out, lse=lse, prefix_len=prefix,
                      prefix_table=None if pt is None else torch.from_numpy(pt).to(DEV))
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_every_token_counts(case, D, fmt):
    """Queries of zero: all weights are the same, and a column's output is the share of its tokens."""
    per, lens, page, prefix, window, sinks = CASES[case]
    if D == 64:                                             # a column's tokens stay below 128, so that one shows
        lens = [min(n, 7000) for n in lens]
    rng = np.random.default_rng(case)
    batch, offsets, lens, table, own, pages, pt = batch_of(per, lens, page, prefix, case)
    shared = T.counting_values(prefix, HKV, D, rng)
    v = [np.concatenate([shared, T.counting_values(int(n) - prefix, HKV, D, rng)]) for n in lens]
    k = [rng.standard_normal(x.shape).astype(np.float32) for x in v]
    cache = cache_of(pool_of(k, table, pages, page, prefix), pool_of(v, table, pages, page, prefix), fmt)
    q = torch.zeros((batch.rows, HQ * D), dtype=torch.bfloat16, device=DEV)
    out, lse = call(q, cache, batch, window, sinks, pt, prefix)
    got = out.double().cpu().numpy().reshape(batch.rows, HQ, D)
    gl = lse.double().cpu().numpy()
    seq, pos = R.positions(offsets, lens, batch.rows)
    for i in range(batch.rows):
        o, l = T.counted(v[seq[i]], int(pos[i]), window, sinks)
        o = o.repeat(HQ // HKV, 0)
        bad = np.abs(got[i] - o) > T.count_tolerance(o)
        assert not bad.any(), (i, seq[i], pos[i], np.argwhere(bad)[:5])
        assert (np.abs(gl[i] - l) <= T.count_lse_tolerance(l)).all(), (i, gl[i], l)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", [i for i, c in enumerate(CASES) if not c[4]])
def test_the_token_that_is_aimed_at(case, D, fmt):
    """A row's key among thousands: its value is the output, so keys and values are of the same tokens."""
    per, lens, page, prefix, _, _ = CASES[case]
    rng = np.random.default_rng(100 + case)
    batch, offsets, lens, table, own, pages, pt = batch_of(per, lens, page, prefix, case)
    q = R.bf16(rng.standard_normal((batch.rows, HQ, D))).float().numpy()
    shared = rng.standard_normal((2, prefix, HKV, D)).astype(np.float32)
    k, v = ([np.concatenate([shared[j], rng.standard_normal((int(n) - prefix, HKV, D)).astype(np.float32)]) for n in lens]
            for j in range(2))
    taken = [set() for _ in range(HKV)]                     # tokens of the prefix, by any sequence
    seq, pos = R.positions(offsets, lens, batch.rows)
    longest = int(np.argmax(lens))
    aims = np.full((batch.rows, HQ), -1)
    for s in range(len(per)):
        mine = slice(offsets[s], offsets[s + 1])
        low = prefix if s % 2 else 0                        # every other sequence's rows aim into the prefix too
        used = [set(x) for x in taken]
        aims[mine] = T.pick_targets(pos[mine], HKV, HQ, rng, low, used)
        for h in range(HKV):
            taken[h] |= {t for t in used[h] if t < prefix}
        into = (aims[mine] >= 0) & (aims[mine] < prefix)
        T.aim(k[longest], q[mine], np.where(into, aims[mine], -1))
        T.aim(k[s], q[mine], np.where(into, -1, aims[mine]))
    for x in k:
        x[:prefix] = k[longest][:prefix]
    cache = cache_of(pool_of(k, table, pages, page, prefix), pool_of(v, table, pages, page, prefix), fmt)
    qd = R.bf16(q.reshape(batch.rows, -1)).to(DEV)
    out, lse = call(qd, cache, batch, 0, 0, pt, prefix)
    check(qd, cache, batch, offsets, lens, own, out, lse, prefix_table=pt, prefix_len=prefix)
    got = out.double().cpu().numpy().reshape(batch.rows, HQ, D)
    kp, vp = R.pool_values(cache)
    scale, group = float(np.float32(D ** -0.5)), HQ // HKV
    o, ref, mag, size = R.attention(q.astype(np.float64), kp, vp, offsets, lens, own, scale, prefix_table=pt,
                                    prefix_len=prefix)
    vmax = np.abs(vp[np.isfinite(vp)]).max()
    tol = R.tolerance(o, mag, size, D, scale, int(max(lens)), vmax)
    for i, h in np.argwhere(aims >= 0):
        t = aims[i, h]
        at = table[longest if t < prefix else seq[i], t // page], h // group, t % page
        # o = w v_t + the others' values times 1 - w in all: |o - v_t| <= (1 - w) (|v_t| + vmax), beside what the
        # definition's own tolerance allows.  (Where many rows aim, their keys meet each other's queries: 1 - w grows.)
        rest = 1.0 - np.exp(scale * q[i, h].astype(np.float64) @ kp[at] - ref[i, h])
        assert rest < 2.0 ** -8
        assert (np.abs(got[i, h] - vp[at]) <= tol[i, h] + rest * (np.abs(vp[at]) + vmax)).all(), (i, h, t)
