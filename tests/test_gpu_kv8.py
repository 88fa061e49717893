"""The 8-bit key/value cache on the GPU: append and read-back bit by bit against the definition, attention against 64
bits within the bound that the other formats are held to (its values are bf16 numbers as well)."""

import numpy as np
import pytest
import torch

import kv8_ref as K
import kv_ref as R
import test_gpu_attention as A
from paper_2606_26587_amd import sharq as S
from test_gpu_kv import CASES, DEV, make_batch, tables

pytestmark = pytest.mark.gpu


def u8(t):
    return t.cpu().view(torch.uint8).numpy()


def pools_of(cache):
    return [u8(t).copy() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]


def filled(pages, page, hkv, D, rule="floor", seed=0, peak=1.0):
    """A cache of tokens that were there before."""
    rng = np.random.default_rng(seed)
    parts = [K.quantize(rng.standard_normal((pages, hkv, page, D)) * peak, rule) for _ in "kv"]
    t = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
    return S.KVCache("fp8", *(t(p[0]).view(torch.float8_e4m3fn) for p in parts), *(t(p[1]) for p in parts),
                     scale_rule=rule)


def append_and_check(per, lens, page, pad, hq, hkv, D, rule="floor", seed=0, peak=0.3, positions=None, angles=None,
                     table_edit=None, x_edit=None, rotate=True):
    batch, offsets, lens, table, pages = make_batch(per, lens, page, pad, seed=seed)
    if table_edit:
        table_edit(table)
        batch.page_table.copy_(torch.from_numpy(table))
    rows, rng = batch.rows, np.random.default_rng(seed)
    x = rng.standard_normal((rows, (hq + 2 * hkv) * D)) * np.exp(rng.standard_normal((rows, 1)))
    if x_edit:
        x_edit(x)
    x = R.bf16(x).to(DEV)
    q, k, v = x[:, :hq * D], x[:, hq * D:(hq + hkv) * D], x[:, (hq + hkv) * D:]
    cos, sin = tables(angles or max(int(lens.max()), 1), D)
    cache = filled(pages, page, hkv, D, rule, seed, peak)
    want = pools_of(cache)
    q_out = torch.full((rows, hq * D), 7.0, dtype=torch.bfloat16, device=DEV)
    pos_t = None if positions is None else torch.tensor(positions, dtype=torch.int32, device=DEV)
    args = (torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV)) if rotate else (None, None)
    S.sharq_kv_append(q if hq else None, k, v, cache, batch, *args, positions=pos_t, q_out=q_out if hq else None)
    torch.cuda.synchronize()

    xs = x.float().cpu().numpy().reshape(rows, hq + 2 * hkv, D)
    seq, pos = R.positions(offsets, lens, rows)
    angle = pos if positions is None else np.array(positions)
    skip = (angle < 0) | (angle >= len(cos)) if rotate else np.zeros(rows, bool)
    at = np.clip(angle, 0, len(cos) - 1)
    y = R.rotate32(xs[:, :hq + hkv], cos[at], sin[at]) if rotate else xs[:, :hq + hkv]
    live = (seq >= 0) & (pos >= 0) & ~skip
    if hq:
        exp = np.where(live[:, None], R.bf16(y[:, :hq].reshape(rows, -1)).float().numpy(), 7.0)
        assert np.array_equal(q_out.float().cpu().numpy(), exp, equal_nan=True)
    K.append(want, y[:, hq:], xs[:, hq + hkv:], offsets, lens, table, page, rule, skip)
    for got, exp, name in zip(pools_of(cache), want, ("k", "v", "k_scale", "v_scale")):
        if len(name) == 1:   # the format has two NaN, 0x7F and 0xFF, and the definition does not say which
            got[got == 0xFF], exp[exp == 0xFF] = 0x7F, 0x7F
        assert np.array_equal(got, exp), (name, np.argwhere(got != exp)[:4], got[got != exp][:4], exp[got != exp][:4])
    return cache, batch, want, table, seq, pos, live


@pytest.mark.parametrize("rule", ["floor", "ceil"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append_and_read(case, D, rule):
    per, lens, page, pad = CASES[case]
    hq, hkv = [(8, 2), (7, 1), (3, 3), (32, 8)][case % 4]
    cache, batch, want, table, seq, pos, _ = append_and_check(per, lens, page, pad, hq, hkv, D, rule, seed=case)
    rows = batch.rows
    k_out = torch.full((rows, hkv * D), 3.0, dtype=torch.bfloat16, device=DEV)
    k_out, v_out = S.sharq_kv_read(cache, batch, k_out=k_out)
    torch.cuda.synchronize()
    for got, codes, scales, name in ((k_out, want[0], want[2], "k"), (v_out, want[1], want[3], "v")):
        val = K.values(codes, scales)
        g = got.double().cpu().numpy().reshape(rows, hkv, D)
        for i in range(rows):
            if seq[i] < 0:
                assert name == "v" or (g[i] == 3.0).all()
            elif pos[i] < 0:
                assert not g[i].any()
            else:
                assert np.array_equal(g[i], val[table[seq[i], pos[i] // page], :, pos[i] % page]), name


@pytest.mark.parametrize("old,new", [(15, 1), (1, 15), (16, 1), (17, 40), (31, 2), (5, 100), (0, 16)])
@pytest.mark.parametrize("peak", [1e-4, 0.3, 50.0])
def test_scales_grow_where_new_tokens_need_it(old, new, peak):
    """Tokens far smaller, smaller and larger than the new ones are there before them."""
    append_and_check([new, 1], [old + new, old + 1], 32, 1, 4, 2, 128, "ceil", seed=old, peak=peak)


def test_appends_one_by_one_are_as_the_definition_says():
    """40 tokens of growing size, one call each, and the same in three calls."""
    rng = np.random.default_rng(2)
    page, hkv, D, n = 32, 2, 64, 40
    x = (rng.standard_normal((n, 2 * hkv * D)) * np.exp2(rng.integers(-9, 4, (n, 1)))).astype(np.float32)
    xt = R.bf16(x).to(DEV)
    xs = xt.float().cpu().numpy().reshape(n, 2 * hkv, D)
    table = np.array([[2, 0]], np.int32)
    tt = torch.from_numpy(table).to(DEV)
    for cuts in (list(range(n + 1)), [0, 7, 8, n]):
        cache = filled(3, page, hkv, D, seed=5)
        want = pools_of(cache)
        for a, b in zip(cuts, cuts[1:]):
            i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
            batch = S.KVBatch(i32(0, b - a), i32(b), tt, b - a, b - a, b)
            S.sharq_kv_append(None, xt[a:b, :hkv * D], xt[a:b, hkv * D:], cache, batch)
            K.append(want, xs[a:b, :hkv], xs[a:b, hkv:], [0, b - a], [b], table, page)
        for got, exp in zip(pools_of(cache), want):
            assert np.array_equal(got, exp)


@pytest.mark.parametrize("new", [1, 5, 40])
def test_rows_that_are_left_out(new):
    """Angles outside the tables: neither query nor key nor value, and the block's scale goes by the others."""
    n = 2 * new
    pos = [(-1, 3, 10 ** 6, 9)[i % 4] for i in range(n + 1)]
    append_and_check([new, new], [new + 9, new], 16, 1, 3, 1, 64, positions=pos, angles=10, seed=new)
    append_and_check([new, new], [new + 9, new], 16, 1, 3, 1, 64, positions=[-5] * (n + 1), angles=10, seed=new)


def test_absent_pages_and_pages_that_end_inside():
    def edit(table):
        table[0, 1], table[1, 0], table[2, 2] = -1, 10 ** 9, -2 ** 31
    append_and_check([40, 3, 70], [60, 3, 75], 16, 2, 2, 2, 128, table_edit=edit, seed=4)
    append_and_check([1, 1, 1], [20, 2, 40], 16, 0, 2, 2, 128, table_edit=edit, seed=5)


def test_values_that_are_not_finite_leave_their_neighbours_alone():
    def edit(x):
        x[2, 300], x[5, 700], x[7, 400], x[7, 401] = np.nan, np.inf, -np.inf, np.nan
        x[9, 256:] = np.inf
    append_and_check([17], [40], 16, 0, 2, 2, 128, x_edit=edit, rotate=False)
    append_and_check([1, 1], [40, 16], 16, 0, 0, 2, 128, x_edit=lambda x: x.__setitem__((0, 3), np.nan), rotate=False)


@pytest.mark.parametrize("rule", ["floor", "ceil"])
def test_magnitudes_from_the_least_to_the_largest(rule):
    def edit(x):
        x *= np.exp2(np.linspace(-140, 120, x.shape[0]))[:, None]
        x[3] = 0
        x[20:40] = -0.0
    append_and_check([200], [203], 64, 0, 1, 1, 128, rule, x_edit=edit, peak=1e-30, rotate=False)


def test_every_code_reads_back():
    page, D = 16, 128
    codes = torch.arange(256, dtype=torch.uint8).repeat(8).view(1, 1, page, D)
    for e in (-117, -50, 0, 3, 119):
        scale = torch.full((1, 1, 1), e + 127, dtype=torch.uint8, device=DEV)
        cache = S.KVCache("fp8", codes.to(DEV).view(torch.float8_e4m3fn), codes.flip(3).contiguous().to(DEV).view(torch.float8_e4m3fn),
                          scale, scale.clone())
        i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
        k, v = S.sharq_kv_read(cache, S.KVBatch(i32(0, 16), i32(16), i32(0)[None], 16, 16, 16))
        for got, t in ((k, cache.k), (v, cache.v)):
            assert np.array_equal(got.double().cpu().numpy(), K.VALUES[u8(t)[0, 0]] * 2.0 ** e, equal_nan=True)


def test_offsets_past_32_bits():
    """Rows at the end of a pool of more than 2^32 bytes of codes."""
    page, hkv, D = 1024, 8, 128
    pages = (2 ** 32 // (page * hkv * D)) + 3
    cache = S.alloc_kv_cache(pages, page, hkv, D, "fp8", DEV)
    rng = np.random.default_rng(0)
    x = R.bf16(rng.standard_normal((40, 2 * hkv * D))).to(DEV)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    batch = S.KVBatch(i32(0, 40), i32(40), i32(pages - 1)[None], 40, 40, 40)
    S.sharq_kv_append(None, x[:, :hkv * D], x[:, hkv * D:], cache, batch)
    k, v = S.sharq_kv_read(cache, batch)
    xs = x.float().cpu().numpy().reshape(40, 2, hkv, D)
    pools = [np.zeros((1, hkv, page, D), np.uint8), np.zeros((1, hkv, page, D), np.uint8),
             np.zeros((1, hkv, page // 16), np.uint8), np.zeros((1, hkv, page // 16), np.uint8)]
    K.append(pools, xs[:, 0], xs[:, 1], [0, 40], [40], [[0]], page)
    for got, c, e in ((k, pools[0], pools[2]), (v, pools[1], pools[3])):
        assert np.array_equal(got.double().cpu().numpy().reshape(40, hkv, D), K.values(c, e)[0, :, :40].swapaxes(0, 1))
    q = R.bf16(rng.standard_normal((40, 16 * D))).to(DEV)
    o = S.sharq_attention(q, cache, batch)
    small = S.KVCache("fp8", *(t[-1:].clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
    o2 = S.sharq_attention(q, small, S.KVBatch(i32(0, 40), i32(40), i32(0)[None], 40, 40, 40))
    assert torch.equal(o, o2)


# ---------------------------------------------------------------------------
# Attention: the cases of the other formats
# ---------------------------------------------------------------------------

@pytest.fixture(autouse=True)
def fp8_in_attention(monkeypatch):
    """Caches of this format for test_gpu_attention's run()."""
    def cache_of(pages, page, hkv, D, fmt, seed=0, peak=1.0):
        rng = np.random.default_rng(seed)
        k = rng.standard_normal((pages, hkv, page, D)) * peak
        v = rng.standard_normal((pages, hkv, page, D)) + rng.standard_normal((1, hkv, 1, D))
        t = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
        parts = [K.quantize(x, "ceil") for x in (k, v)]
        return S.KVCache("fp8", *(t(p[0]).view(torch.float8_e4m3fn) for p in parts), *(t(p[1]) for p in parts))

    def poison(cache, seen):
        m = torch.from_numpy(~seen).to(DEV)[:, None, :].expand(-1, cache.kv_heads, -1)
        b = torch.from_numpy(~seen.reshape(seen.shape[0], -1, 16).any(-1)).to(DEV)[:, None].expand(-1, cache.kv_heads, -1)
        for t in (cache.k, cache.v):
            t.view(torch.uint8)[m] = 0x7F
        for t in (cache.k_scale, cache.v_scale):
            t[b] = 0xFF

    monkeypatch.setattr(A, "filled_cache", cache_of)
    monkeypatch.setattr(A, "poison", poison)
    monkeypatch.setattr(R, "pool_values", K.pool_values)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 300, 1025])
def test_single_token(n, D):
    A.run([1], [n], 16, 8, 2, D, "fp8", seed=n)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 4), (7, 1), (16, 1), (12, 3), (28, 4), (32, 1), (64, 1), (128, 1)])
def test_decode_batch(hq, hkv, D):
    lens = [1, 700, 64, 65, 3, 0, 128, 257, 33]
    A.run([1] * 5 + [0] + [1] * 3, lens, 32, hq, hkv, D, "fp8", pad=2, seed=hq)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts(D, page):
    A.run([33, 1, 130, 64], [33, 1, 130, 64], page, 4, 2, D, "fp8", pad=3, seed=page)


@pytest.mark.parametrize("per,lens", [([5, 40], [100, 333]), ([1, 70, 0, 3], [400, 71, 9, 3]),
                                      ([4, 4, 4], [4, 100, 259]), ([20, 2], [19, 1])])
def test_chunks_over_cached_tokens(per, lens):
    A.run(per, lens, 16, 6, 2, 128, "fp8", seed=lens[0])


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (64, 0), (65, 100), (200, 1), (10 ** 6, 4),
                                          (50, 10 ** 6), (2 ** 40, 2 ** 40)])
def test_window_and_sinks(window, sinks):
    A.run([1, 90, 5], [500, 90, 321], 16, 4, 1, 64, "fp8", window=window, sinks=sinks, seed=window % 97)


def test_long_window():
    A.run([1, 1, 3], [2500, 1300, 4100], 64, 8, 2, 128, "fp8", window=1024, sinks=4)


@pytest.mark.parametrize("per,lens,prefix,window,sinks", [
    ([1] * 5, [65, 80, 64, 129, 300], 64, 0, 0),
    ([1] * 40, [520 + 3 * i for i in range(40)], 512, 0, 0),
    ([3, 1, 4], [200, 150, 131], 128, 0, 0),
    ([1] * 5, [400, 333, 280, 500, 290], 256, 100, 8),
    ([70, 1, 2], [90, 65, 70], 64, 0, 0),
    ([16, 2], [16, 70], 64, 0, 0),
    ([0, 1, 1], [0, 90, 100], 64, 0, 0),
])
def test_shared_prefix(per, lens, prefix, window, sinks):
    A.run(per, lens, 16, 8, 2, 128, "fp8", window=window, sinks=sinks, prefix_len=prefix, pad=1, seed=prefix)


@pytest.mark.parametrize("D", [64, 128])
def test_shared_prefix_heads(D):
    A.run([2] * 20, [300 + 7 * i for i in range(20)], 32, 7, 1, D, "fp8", prefix_len=256)


def test_absent_pages():
    A.run([1, 40], [200, 100], 16, 4, 2, 128, "fp8", bad_pages=[(0, 0, -1), (0, 7, 3), (1, 2, -5), (1, 6, 0)])
    A.run([2], [20], 16, 4, 2, 128, "fp8", bad_pages=[(0, 0, -1), (0, 1, -1)])


@pytest.mark.parametrize("per,lens", [([1], [900]), ([100], [100])])
def test_large_scores(per, lens):
    A.run(per, lens, 16, 4, 2, 128, "fp8", peak=6.0)


@pytest.mark.parametrize("D", [64, 128])
def test_prompts_and_single_tokens_in_one_launch(D):
    """A long prompt and single tokens, unsplit: both kernels in one launch."""
    A.run([200] + [1] * 40, [200] + [17 * i + 1 for i in range(40)], 16, 8, 8, D, "fp8", seed=1)


def test_a_nan_that_a_row_sees():
    batch, offsets, lens, table, pages = make_batch([1, 60], [100, 60], 16)
    cache = filled(pages, 16, 2, 128)
    cache.k.view(torch.uint8)[table[0, 3], 0, 5, 7] = 0x7F
    cache.v.view(torch.uint8)[table[1, 2], 1, 9, 11] = 0xFF
    q = R.bf16(np.random.default_rng(0).standard_normal((batch.rows, 8 * 128))).to(DEV)
    o = S.sharq_attention(q, cache, batch).float().view(61, 8, 128)
    assert o[0, :4].isnan().all() and not o[0, 4:].isnan().any()
    assert o[1 + 41:, 4:, 11].isnan().all() and not o[1:, :4].isnan().any()
    o[1:, 4:, 11] = 0
    assert not o[1:, 4:].isnan().any()
