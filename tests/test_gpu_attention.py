"""Attention over the paged key/value cache on the GPU against the definition
in 64 bits, within a bound that is derived from the roundings it makes."""

import numpy as np
import pytest
import torch

import kv_ref as R
from paper_2606_26587_amd import sharq as S
from test_gpu_kv import DEV, make_batch

pytestmark = pytest.mark.gpu


def filled_cache(pages, page, hkv, D, fmt, seed=0, peak=1.0):
    rng = np.random.default_rng(seed)
    shape = (pages, hkv, page, D)
    k = (rng.standard_normal(shape) * peak).astype(np.float32)
    v = (rng.standard_normal(shape) + rng.standard_normal((1, hkv, 1, D))).astype(np.float32)
    if fmt == "bf16":
        return S.KVCache(fmt, R.bf16(k).to(DEV), R.bf16(v).to(DEV))
    parts = []
    for x in (k, v):
        c, e = R.mx_quantize(x)
        parts.append((torch.from_numpy(c[..., 0::2] | c[..., 1::2] << 4).to(DEV), torch.from_numpy(e).to(DEV)))
    return S.KVCache(fmt, parts[0][0], parts[1][0], parts[0][1], parts[1][1])


def spoil(cache, table, lens, page, low=None, sinks=0, prefix_len=0):
    """NaN into every slot that no sequence's visible tokens occupy."""
    seen = np.zeros((cache.pages, page), bool)
    for s, n in enumerate(lens):
        for t in range(prefix_len, max(int(n), 0)):
            pg = table[s, t // page]
            if 0 <= pg < cache.pages and (low is None or t >= low[s] or t < sinks):
                seen[pg, t % page] = True
    return seen


def poison(cache, seen):
    m = torch.from_numpy(~seen).to(DEV)[:, None, :].expand(-1, cache.kv_heads, -1)
    if cache.fmt == "bf16":
        cache.k[m] = float("nan")
        cache.v[m] = float("inf")
    else:
        for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
            t[m] = 0xFF


def check(q, cache, batch, offsets, lens, table, out, lse, window=0, sinks=0, prefix_table=None, prefix_len=0,
          scale=None):
    D, rows = cache.head_dim, batch.rows
    scale = D ** -0.5 if scale is None else scale
    scale = float(np.float32(scale))
    kp, vp = R.pool_values(cache)
    qd = q.double().cpu().numpy().reshape(rows, -1, D)
    o, l, mag, size = R.attention(qd, kp, vp, offsets, lens, table, scale, window, sinks, prefix_table, prefix_len)
    n = int(max(list(lens) + [0]))
    live = ~np.isnan(l[:, 0])
    got = out.double().cpu().numpy().reshape(o.shape)
    tol = R.tolerance(o, mag, size, D, scale, n, np.abs(vp[np.isfinite(vp)]).max(initial=0.0))
    bad = np.abs(got - o)[live] > tol[live]
    assert not bad.any(), (bad.mean(), np.abs(got - o)[live].max())
    assert (got[~live] == 9.0).all()                        # padding rows stay
    gl = lse.double().cpu().numpy()
    empty = live[:, None] & np.isneginf(l)
    assert np.isneginf(gl[empty]).all() and (got[empty] == 0).all()
    fine = live[:, None] & np.isfinite(l)
    assert (np.abs(gl[fine] - l[fine]) <= R.lse_tolerance(l, size, D, scale, n)[fine]).all()
    assert (gl[~live] == 9.0).all()


def run(per, lens, page, hq, hkv, D, fmt, window=0, sinks=0, pad=0, seed=0, prefix_len=0, bad_pages=(), peak=1.0,
        scale=None):
    batch, offsets, lens, table, pages = make_batch(per, lens, page, pad, seed=seed)
    for s, j, value in bad_pages:
        table[s, j] = value if value < 0 else pages + value
    prefix = None
    if prefix_len:
        prefix = table[int(np.argmax(lens)), :prefix_len // page].copy()
        table[:, :prefix_len // page] = 10 ** 6             # not looked at
    batch.page_table.copy_(torch.from_numpy(table))
    cache = filled_cache(pages, page, hkv, D, fmt, seed, peak)
    low = None
    if window:
        low = [max(0, int(lens[s]) - per[s] - window + 1) for s in range(len(per))]
    seen = spoil(cache, table, lens, page, low, sinks, prefix_len)
    if prefix_len:
        for t in range(min(prefix_len, int(max(lens)))):
            seen[prefix[t // page], t % page] = True
    poison(cache, seen)
    rng = np.random.default_rng(seed + 1)
    q = R.bf16(rng.standard_normal((batch.rows, hq * D)) * peak).to(DEV)
    out = torch.full((batch.rows, hq * D), 9.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((batch.rows, hq), 9.0, dtype=torch.float32, device=DEV)
    pt = None if prefix is None else torch.from_numpy(prefix).to(DEV)
    S.sharq_attention(q, cache, batch, scale=scale, window=window, sinks=sinks, prefix_table=pt, prefix_len=prefix_len,
                      out=out, lse=lse)
    torch.cuda.synchronize()
    # the poisoned slots are out of every row's sight: the definition never touches them
    if fmt == "mx":
        for e in (cache.k_scale, cache.v_scale):
            e[e == 0xFF] = 0
    check(q, cache, batch, offsets, lens, table, out, lse, window, sinks, prefix, prefix_len, scale)


FMTS = ["bf16", "mx"]


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 300, 1025])
def test_single_token(n, D, fmt):
    run([1], [n], 16, 8, 2, D, fmt, seed=n)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("hq,hkv", [(4, 4), (7, 1), (16, 1), (12, 3), (28, 4), (64, 1), (128, 1)])
def test_decode_batch(hq, hkv, fmt):
    lens = [1, 700, 64, 65, 3, 0, 128, 257, 33]
    run([1] * 5 + [0] + [1] * 3, lens, 32, hq, hkv, 128, fmt, pad=2, seed=hq)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts(D, page, fmt):
    run([33, 1, 130, 64], [33, 1, 130, 64], page, 4, 2, D, fmt, pad=3, seed=page)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("per,lens", [([5, 40], [100, 333]), ([1, 70, 0, 3], [400, 71, 9, 3]),
                                      ([4, 4, 4], [4, 100, 259]), ([20, 2], [19, 1])])
def test_chunks_over_cached_tokens(per, lens, fmt):
    run(per, lens, 16, 6, 2, 128, fmt, seed=lens[0])


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (64, 0), (65, 100), (200, 1), (10 ** 6, 4),
                                          (50, 10 ** 6), (2 ** 40, 2 ** 40)])
def test_window_and_sinks(window, sinks, fmt):
    run([1, 90, 5], [500, 90, 321], 16, 4, 1, 64, fmt, window=window, sinks=sinks, seed=window % 97)


@pytest.mark.parametrize("fmt", FMTS)
def test_long_window(fmt):
    run([1, 1, 3], [2500, 1300, 4100], 64, 8, 2, 128, fmt, window=1024, sinks=4)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("per,lens,prefix,window,sinks", [
    ([1] * 5, [65, 80, 64, 129, 300], 64, 0, 0),      # one sequence is the prefix alone
    ([1] * 40, [520 + 3 * i for i in range(40)], 512, 0, 0),
    ([3, 1, 4], [200, 150, 131], 128, 0, 0),
    ([1] * 5, [400, 333, 280, 500, 290], 256, 100, 8),  # the window leaves most of the prefix
    ([1] * 3, [400, 333, 280], 256, 50, 0),
    ([70, 1, 2], [90, 65, 70], 64, 0, 0),
    ([16, 2], [16, 70], 64, 0, 0),                    # a sequence that ends inside the prefix
    ([0, 1, 1], [0, 90, 100], 64, 0, 0),
])
def test_shared_prefix(per, lens, prefix, window, sinks, fmt):
    run(per, lens, 16, 8, 2, 128, fmt, window=window, sinks=sinks, prefix_len=prefix, pad=1, seed=prefix)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("D", [64, 128])
def test_shared_prefix_heads(D, fmt):
    run([2] * 20, [300 + 7 * i for i in range(20)], 32, 7, 1, D, fmt, prefix_len=256)


@pytest.mark.parametrize("fmt", FMTS)
def test_absent_pages(fmt):
    run([1, 40], [200, 100], 16, 4, 2, 128, fmt, bad_pages=[(0, 0, -1), (0, 7, 3), (1, 2, -5), (1, 6, 0)])
    run([2], [20], 16, 4, 2, 128, fmt, bad_pages=[(0, 0, -1), (0, 1, -1)])   # nothing is left


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("per,lens", [([1], [900]), ([100], [100])])
def test_large_scores(per, lens, fmt):
    """Scores in the hundreds: one token takes all the weight."""
    run(per, lens, 16, 4, 1, 128, fmt, peak=6.0, scale=1.0)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("per,lens,prefix", [([1], [9000], 0), ([1, 3, 2], [6000, 10, 3500], 0), ([9], [5000], 0),
                                             ([30, 18], [3000, 700], 0), ([1] * 3, [5000, 4100, 4500], 4096),
                                             ([25, 1], [2300, 2100], 2048)])
def test_tokens_split_over_workgroups(per, lens, prefix, D, fmt):
    run(per, lens, 64, 8, 2, D, fmt, prefix_len=prefix, pad=1, seed=len(per))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("per", [1, 40])
def test_large_scale_where_a_wavefront_sees_nothing(per, fmt):
    """The running maximum's start times a scale above 1 is not a number that may enter a sum."""
    run([per], [500], 16, 4, 1, 128, fmt, scale=3.0, bad_pages=[(0, j, -1) for j in range(24)], peak=0.3)
    run([per, per], [per, 70], 16, 4, 1, 128, fmt, scale=3.0, window=20, prefix_len=32, peak=0.3)
