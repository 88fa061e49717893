"""Paged key/value cache on the GPU: the append (rotation, bf16 and MXFP4
storage) and the read-back, bit by bit against the definition."""

import numpy as np
import pytest
import torch

import kv_ref as R
from paper_2606_26587_amd import sharq as S

pytestmark = pytest.mark.gpu
DEV = "cuda"


def make_batch(rows_per_seq, lens, page, pad=0, spare=2, seed=0, extra_pages=3):
    """A KVBatch with shuffled pages; returns (batch, offsets, lens, table) with numpy copies."""
    rng = np.random.default_rng(seed)
    need = [-(-n // page) for n in lens]
    ids = rng.permutation(sum(need) + extra_pages)
    table = np.full((len(lens), max(need + [0]) + spare), 10 ** 6, np.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = ids[at:at + n]
        at += n
    offsets = np.concatenate([[0], np.cumsum(rows_per_seq)]).astype(np.int32)
    rows = int(offsets[-1]) + pad
    lens = np.array(lens, np.int32)
    dev = [torch.from_numpy(x).to(DEV) for x in (offsets, lens, table)]
    batch = S.KVBatch(*dev, rows, max(list(rows_per_seq) + [0]), int(max(list(lens) + [0])))
    return batch, offsets, lens, table, sum(need) + extra_pages


def empty_cache(pages, page, hkv, D, fmt, rule="floor"):
    """A cache whose slots hold a pattern that no append writes by chance."""
    c = S.alloc_kv_cache(pages, page, hkv, D, fmt, DEV, rule)
    for t in (c.k, c.v, c.k_scale, c.v_scale):
        if t is not None:
            t.view(torch.uint8).fill_(0x5A)
    return c


def tables(n, D):
    a = np.arange(n)[:, None] * 10000.0 ** (-2.0 * np.arange(D // 2) / D)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def expected_pools(cache_before, k, v, seq, pos, table, skip, pages, page, fmt, rule):
    """The pools' bytes after the append of fp32 rows k, v [rows, heads, D]."""
    out = [None if t is None else t.cpu().view(torch.uint8).numpy().copy() for t in cache_before]
    for i in range(len(seq)):
        if seq[i] < 0 or pos[i] < 0 or skip[i]:
            continue
        pg = table[seq[i], pos[i] // page]
        if not 0 <= pg < pages:
            continue
        for j, x in enumerate((k[i], v[i])):
            if fmt == "bf16":
                out[j][pg, :, pos[i] % page] = R.bf16(x).view(torch.uint8).numpy()
            else:
                c, e = R.mx_quantize(x, rule)
                out[j][pg, :, pos[i] % page] = c[:, 0::2] | c[:, 1::2] << 4
                out[2 + j][pg, :, pos[i] % page] = e
    return out


CASES = [
    # rows per sequence, lengths, page, padding rows
    ([1], [1], 16, 0),
    ([1], [33], 16, 3),
    ([5], [5], 16, 0),
    ([1, 0, 7, 2], [40, 0, 7, 1000], 32, 2),        # an empty sequence, long and short ones
    ([3, 4], [2, 70], 64, 1),                       # more rows than tokens: a row at a negative position
    ([130], [200], 1024, 0),
    ([1] * 70, list(range(1, 71)), 16, 0),          # more sequences than a wavefront
    ([0, 1, 0, 0, 2] * 60, [5, 9, 0, 1, 30] * 60, 16, 5),
]


@pytest.mark.parametrize("fmt", ["bf16", "mx"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_append_and_read(case, D, fmt):
    per, lens, page, pad = CASES[case]
    hq, hkv = [(8, 2), (7, 1), (3, 3), (32, 8)][case % 4]
    batch, offsets, lens, table, pages = make_batch(per, lens, page, pad, seed=case)
    rows = batch.rows
    rng = np.random.default_rng(case)
    x = R.bf16(rng.standard_normal((rows, (hq + 2 * hkv) * D)) * np.exp(rng.standard_normal((rows, 1)))).to(DEV)
    q, k, v = x[:, :hq * D], x[:, hq * D:(hq + hkv) * D], x[:, (hq + hkv) * D:]
    cos, sin = tables(max(int(lens.max()), 1), D)
    cache = empty_cache(pages, page, hkv, D, fmt)
    before = [None if t is None else t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    q_out = torch.full((rows, hq * D), 7.0, dtype=torch.bfloat16, device=DEV)
    S.sharq_kv_append(q, k, v, cache, batch, torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV), q_out=q_out)
    torch.cuda.synchronize()

    xs = x.float().cpu().numpy().reshape(rows, hq + 2 * hkv, D)
    seq, pos = R.positions(offsets, lens, rows)
    at = np.clip(pos, 0, None)
    y = R.rotate32(xs[:, :hq + hkv], cos[at], sin[at])
    live = (seq >= 0) & (pos >= 0)
    want = np.where(live[:, None], R.bf16(y[:, :hq].reshape(rows, -1)).float().numpy(), 7.0)
    assert np.array_equal(q_out.float().cpu().numpy(), want)
    pools = expected_pools(before, y[:, hq:], xs[:, hq + hkv:], seq, pos, table, np.zeros(rows, bool), pages, page, fmt,
                           "floor")
    for got, exp in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), pools):
        if exp is not None:
            assert np.array_equal(got.cpu().view(torch.uint8).numpy(), exp)

    k_out = torch.full((rows, hkv * D), 3.0, dtype=torch.bfloat16, device=DEV)
    k_out, v_out = S.sharq_kv_read(cache, batch, k_out=k_out)
    torch.cuda.synchronize()
    for got, src, name in ((k_out, y[:, hq:], "k"), (v_out, xs[:, hq + hkv:], "v")):
        val = R.bf16(src).double().numpy() if fmt == "bf16" else R.mx_values(*R.mx_quantize(src))
        val = val.reshape(rows, -1)
        g = got.double().cpu().numpy()
        assert np.array_equal(g[live], val[live]), name
        assert not g[(seq >= 0) & (pos < 0)].any()          # a row without a token reads as zeros
        if name == "k":
            assert (g[seq < 0] == 3.0).all()                # padding rows stay


@pytest.mark.parametrize("fmt", ["bf16", "mx"])
def test_append_in_place_positions_no_rotation_and_values_alone(fmt):
    D, hq, hkv, page = 128, 4, 2, 16
    batch, offsets, lens, table, pages = make_batch([3, 2], [20, 9], page, 1)
    rows = batch.rows
    rng = np.random.default_rng(5)
    x0 = R.bf16(rng.standard_normal((rows, (hq + 2 * hkv) * D)))
    cos, sin = tables(50, D)
    dc, ds = torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV)
    where = np.array([49, 0, 50, -1, 7, 3], np.int32)       # two angles outside the tables, one row of padding
    x = x0.to(DEV)
    cache = empty_cache(pages, page, hkv, D, fmt)
    before = [None if t is None else t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    q, k, v = x[:, :hq * D], x[:, hq * D:(hq + hkv) * D], x[:, (hq + hkv) * D:]
    assert S.sharq_kv_append(q, k, v, cache, batch, dc, ds, positions=torch.from_numpy(where).to(DEV), q_out=q) is q
    xs = x0.float().numpy().reshape(rows, -1, D)
    seq, pos = R.positions(offsets, lens, rows)
    out = (where < 0) | (where >= 50)
    at = np.clip(where, 0, 49)
    y = R.rotate32(xs[:, :hq + hkv], cos[at], sin[at])
    keep = out | (seq < 0)
    want = np.where(keep[:, None], xs[:, :hq].reshape(rows, -1), R.bf16(y[:, :hq].reshape(rows, -1)).float().numpy())
    assert np.array_equal(q.float().cpu().numpy(), want)
    assert torch.equal(x[:, hq * D:].cpu(), x0[:, hq * D:])
    pools = expected_pools(before, y[:, hq:], xs[:, hq + hkv:], seq, pos, table, out, pages, page, fmt, "floor")
    for got, exp in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), pools):
        assert exp is None or np.array_equal(got.cpu().view(torch.uint8).numpy(), exp)
    # without tables nothing turns; without queries only the cache is written
    cache = empty_cache(pages, page, hkv, D, fmt)
    assert S.sharq_kv_append(None, k, v, cache, batch) is None
    pools = expected_pools(before, xs[:, hq:hq + hkv], xs[:, hq + hkv:], seq, pos, table, np.zeros(rows, bool), pages,
                           page, fmt, "floor")
    for got, exp in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), pools):
        assert exp is None or np.array_equal(got.cpu().view(torch.uint8).numpy(), exp)


@pytest.mark.parametrize("rule", ["floor", "ceil"])
def test_mx_blocks_of_all_sizes(rule):
    """Zeros, subnormals, ties of the grid, the largest values, every exponent."""
    D, hkv, page = 64, 1, 16
    rng = np.random.default_rng(2)
    rows = 300
    x = rng.standard_normal((rows, D)).astype(np.float32)
    x *= np.exp2(np.linspace(-140, 125, rows)).astype(np.float32)[:, None]
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 7.5, 0.0, -0.0, -0.25, -5.0, -3.5, 4.0], np.float32)
    for i in range(0, rows, 3):
        x[i] = np.tile(ties, D // 16) * np.float32(2.0) ** (i // 3 - 50)
    x[1] = 0.0
    x[2, :32] = -0.0
    kb = R.bf16(x)
    batch, offsets, lens, table, pages = make_batch([rows], [rows], page)
    cache = empty_cache(pages, page, hkv, D, "mx", rule)
    S.sharq_kv_append(None, kb.to(DEV), kb.to(DEV), cache, batch)
    k, v = S.sharq_kv_read(cache, batch)
    codes, scales = R.mx_quantize(kb.float().numpy(), rule)
    seq, pos = R.positions(offsets, lens, rows)
    pg, sl = table[0, pos // page], pos % page
    for t, e in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        assert np.array_equal(e.cpu().numpy()[pg, 0, sl], scales)
        assert np.array_equal(R.unpack(t.cpu().numpy()[pg, 0, sl]), codes)
    assert np.array_equal(k.double().cpu().numpy(), R.mx_values(codes, scales))
    assert torch.equal(k, v)


@pytest.mark.parametrize("fmt", ["bf16", "mx"])
def test_absent_pages_and_wild_offsets_stay_in_bounds(fmt):
    """Page table entries outside the pool store nothing and read as zeros; offsets and lengths that break the
    contract (decreasing, beyond the rows, beyond max_len) reach no memory outside the buffers."""
    D, hkv, page = 128, 2, 16
    batch, offsets, lens, table, pages = make_batch([4, 40], [4, 60], page, 2)
    bad = table.copy()
    bad[1, 1], bad[1, 2] = -1, pages
    batch.page_table.copy_(torch.from_numpy(bad))
    rows = batch.rows
    x = R.bf16(np.random.default_rng(1).standard_normal((rows, hkv * D))).to(DEV)
    cache = empty_cache(pages, page, hkv, D, fmt)
    before = [None if t is None else t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    S.sharq_kv_append(None, x, x, cache, batch)
    xs = x.float().cpu().numpy().reshape(rows, hkv, D)
    seq, pos = R.positions(offsets, lens, rows)
    pools = expected_pools(before, xs, xs, seq, pos, bad, np.zeros(rows, bool), pages, page, fmt, "floor")
    for got, exp in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), pools):
        assert exp is None or np.array_equal(got.cpu().view(torch.uint8).numpy(), exp)
    k, v = S.sharq_kv_read(cache, batch)
    gone = (seq == 1) & (pos >= page) & (pos < 3 * page)
    assert gone.any() and not k.cpu()[torch.from_numpy(gone)].any() and not v.cpu()[torch.from_numpy(gone)].any()
    for o, l in (([0, 50, 20], [4, 60]), ([-7, 3, 2 ** 31 - 1], [2 ** 31 - 1, -5]), ([46, 0, 46], [10 ** 9, 10 ** 9])):
        batch.row_offsets.copy_(torch.tensor(o, dtype=torch.int32))
        batch.lens.copy_(torch.tensor(l, dtype=torch.int32))
        S.sharq_kv_append(None, x, x, cache, batch)
        S.sharq_kv_read(cache, batch, k, v)
    torch.cuda.synchronize()
