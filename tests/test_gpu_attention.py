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


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("per,lens,prefix", [([1, 1], [3000, 20], 0), ([70], [90], 0), ([2, 1], [300, 600], 256)])
@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** -60])
def test_smallest_scales(scale, per, lens, prefix, fmt):
    """Scores of nearly nothing: the outputs are means of the visible values."""
    run(per, lens, 16, 4, 2, 128, fmt, scale=scale, prefix_len=prefix)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("prefix", [0, 192])
@pytest.mark.parametrize("new", [1, 4, 5, 8, 9, 16, 17, 33])
def test_rows_around_the_limits_of_the_kernels(new, prefix, D, fmt):
    """16, 32, 64 and 128 rows of a sequence and key/value head and one token more, with 4 query heads to a head."""
    run([new, max(1, new - 3), 1], [700, 260, 450], 16, 8, 2, D, fmt, prefix_len=prefix)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("D,hkv,group", [(128, 8, 4), (64, 16, 4), (128, 8, 1), (128, 4, 16), (64, 16, 17)])
@pytest.mark.parametrize("window,sinks,prefix", [(0, 0, 0), (37, 3, 0), (50, 0, 48)])
def test_prompts_and_single_tokens_in_one_call(window, sinks, prefix, D, hkv, group, fmt):
    """Many sequences of one or a few rows beside some of many: on an MXFP4 cache each kind has its kernel, in one launch."""
    new = [150, 1, 0, 4, 5, 1, 16, 17, 1, 64] + [1] * 60
    lens = [150, 200, 80, 90, 5, 1, 130, 70, 64, 300] + [48 + 3 * i for i in range(60)]
    if prefix:
        lens = [max(n, prefix + 1) for n in lens]
    table_of = dict(bad_pages=[(1, 2, -1), (12, 0, 0)]) if not prefix else {}
    run(new, lens, 16, hkv * group, hkv, D, fmt, window=window, sinks=sinks, prefix_len=prefix, pad=11, **table_of)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("count", [65, 130, 200])
def test_more_sequences_than_a_wavefront(count, fmt):
    rng = np.random.default_rng(count)
    lens = [int(x) for x in rng.integers(0, 90, count)]
    run([min(n, 1) for n in lens], lens, 16, 4, 2, 64, fmt, pad=3, seed=count)
    per = [int(rng.integers(0, n + 1)) for n in lens]
    per[7], lens[7] = 40, 60                            # (more rows than the kernel for few rows takes)
    run(per, lens, 16, 4, 2, 64, fmt, pad=3, seed=count)
    lens = [64 + n for n in lens]
    run([1] * count, lens, 16, 8, 2, 64, fmt, prefix_len=64, seed=count)
    run([int(x) for x in rng.integers(0, 40, count)], lens, 16, 2, 1, 64, fmt, prefix_len=64, seed=count)


def setup(per, lens, page, hq, hkv, D, fmt, slack=0, more_rows=0, pad=0, seed=3):
    batch, offsets, lens, table, pages = make_batch(per, lens, page, pad, spare=2 + slack // page, seed=seed)
    if slack or more_rows:
        batch = S.KVBatch(batch.row_offsets, batch.lens, batch.page_table, batch.rows, batch.max_rows + more_rows,
                          batch.max_len + slack)
    cache = filled_cache(pages, page, hkv, D, fmt, seed)
    q = R.bf16(np.random.default_rng(seed).standard_normal((batch.rows, hq * D))).to(DEV)
    return batch, offsets, lens, table, cache, q


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("per,lens", [([1, 1], [300, 40]), ([50, 3], [300, 40])])
def test_loose_bounds_of_the_batch(per, lens, fmt):
    """max_len and max_rows bound the sequences; how far above they are changes the split, not the result."""
    for slack, more in ((0, 0), (160, 0), (16000, 3), (16, 100)):
        batch, offsets, ln, table, cache, q = setup(per, lens, 16, 4, 2, 128, fmt, slack, more)
        out = torch.full((batch.rows, 4 * 128), 9.0, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((batch.rows, 4), 9.0, device=DEV)
        S.sharq_attention(q, cache, batch, out=out, lse=lse)
        check(q, cache, batch, offsets, ln, table, out, lse)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("per,lens,prefix", [([1], [3000], 0), ([1, 1], [900, 1500], 256), ([5, 2], [3000, 40], 0),
                                             ([200], [1500], 0)])
def test_many_padding_rows(per, lens, prefix, fmt):
    """More rows than the sequences can own: the workspace is that of the call without them, and they stay as they are."""
    batch, offsets, ln, table, cache, q = setup(per, lens, 16, 4, 2, 128, fmt)
    pt = batch.page_table[0, :prefix // 16].contiguous() if prefix else None
    q = q[:sum(per)]
    rows = len(per) * max(per) + 1000
    wide = S.KVBatch(batch.row_offsets, batch.lens, batch.page_table, rows, max(per), batch.max_len)
    qw = torch.full((rows, 512), float("nan"), dtype=torch.bfloat16, device=DEV)
    qw[:sum(per)] = q
    out = torch.full((rows, 512), 9.0, dtype=torch.bfloat16, device=DEV)
    lw = torch.full((rows, 4), 9.0, device=DEV)
    most = S.KVBatch(batch.row_offsets, batch.lens, batch.page_table, len(per) * max(per), max(per), batch.max_len)
    size = S.attention_workspace_bytes(cache, wide, 4, prefix_len=prefix)
    assert size == S.attention_workspace_bytes(cache, most, 4, prefix_len=prefix)
    ws = torch.full((size + 256,), 255, dtype=torch.uint8, device=DEV)
    S.sharq_attention(qw, cache, wide, prefix_table=pt, prefix_len=prefix, out=out, lse=lw, workspace=ws[:size])
    assert (ws[size:] == 255).all() and (out[sum(per):] == 9).all() and (lw[sum(per):] == 9).all()
    bare = S.KVBatch(batch.row_offsets, batch.lens, batch.page_table, sum(per), max(per), batch.max_len)
    check(q, cache, bare, offsets, ln, table, out[:sum(per)], lw[:sum(per)], prefix_len=prefix,
          prefix_table=None if pt is None else pt.cpu().numpy())


@pytest.mark.parametrize("fmt", FMTS)
def test_strided_rows_default_output_and_repeated_calls(fmt):
    per, lens = [1, 1, 1, 2], [4000, 17, 256, 2000]
    batch, offsets, ln, table, cache, q = setup(per, lens, 64, 8, 2, 128, fmt)
    wide = torch.zeros((batch.rows, 8 * 128 + 64), dtype=torch.bfloat16, device=DEV)
    wide[:, 32:-32] = q
    first = S.sharq_attention(q, cache, batch)
    again = S.sharq_attention(wide[:, 32:-32], cache, batch, out=wide[:, 32:-32].clone())
    assert torch.equal(first, again)
    outw = torch.full_like(wide, 5.0)
    S.sharq_attention(wide[:, 32:-32], cache, batch, out=outw[:, 32:-32])
    assert torch.equal(outw[:, 32:-32], first) and (outw[:, :32] == 5).all() and (outw[:, -32:] == 5).all()
    # the table as a slice of a wider one, and a workspace full of NaN
    big = torch.full((4, 200), -1, dtype=torch.int32, device=DEV)
    big[:, :table.shape[1]] = batch.page_table
    sliced = S.KVBatch(batch.row_offsets, batch.lens, big[:, :table.shape[1] + 1], batch.rows, batch.max_rows, batch.max_len)
    ws = torch.full((S.attention_workspace_bytes(cache, sliced, 8),), 255, dtype=torch.uint8, device=DEV)
    assert ws.numel() > 0
    assert torch.equal(S.sharq_attention(q, cache, sliced, workspace=ws), first)
    with pytest.raises(S.SharqError):
        S.sharq_attention(q, cache, sliced, workspace=ws[:-16])


@pytest.mark.parametrize("fmt", FMTS)
def test_streams_and_graphs(fmt):
    """A call on a stream of its own, and one captured decode step (append, attention, behind a shared prefix too)
    replayed on changed inputs, with eager calls between the replays."""
    per, lens, page, hq, hkv, D = [1] * 6, [300, 290, 4000, 256, 257, 310], 64, 8, 2, 128
    batch, offsets, ln, table, cache, q = setup(per, lens, page, hq, hkv, D, fmt)
    rows = batch.rows
    gen = torch.Generator(device=DEV).manual_seed(0)
    x = torch.randn((rows, (hq + 2 * hkv) * D), generator=gen, device=DEV).to(torch.bfloat16)
    cos, sin = (torch.from_numpy(t).to(DEV) for t in np_tables(5000, D))
    pt = batch.page_table[2, :4].contiguous()
    q_out, out, out2 = (torch.zeros((rows, hq * D), dtype=torch.bfloat16, device=DEV) for _ in range(3))
    ws = torch.empty(max(S.attention_workspace_bytes(cache, batch, hq),
                         S.attention_workspace_bytes(cache, batch, hq, prefix_len=256)), dtype=torch.uint8, device=DEV)

    def step(stream=None):
        w = hq * D, (hq + hkv) * D
        S.sharq_kv_append(x[:, :w[0]], x[:, w[0]:w[1]], x[:, w[1]:], cache, batch, cos, sin, q_out=q_out, stream=stream)
        S.sharq_attention(q_out, cache, batch, out=out, workspace=ws, stream=stream)
        S.sharq_attention(q_out, cache, batch, prefix_table=pt, prefix_len=256, out=out2, workspace=ws, stream=stream)

    step()
    torch.cuda.synchronize()
    want, want2 = out.clone(), out2.clone()
    side = torch.cuda.Stream()
    out.zero_()
    out2.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    # (a workspace that the call allocates itself is taken on that stream)
    mine = S.sharq_attention(q_out, cache, batch, stream=side, out=torch.empty_like(out))
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(out2, want2) and torch.equal(mine, want)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(torch.randn(x.shape, generator=gen, device=DEV))
        batch.lens.copy_(torch.tensor([n - i for n in lens], dtype=torch.int32))
        out.zero_()
        out2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got, got2, pools = out.clone(), out2.clone(), (cache.k.clone(), cache.v.clone())
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(got2, out2)
        assert torch.equal(pools[0].view(torch.uint8), cache.k.view(torch.uint8))
        assert torch.equal(pools[1].view(torch.uint8), cache.v.view(torch.uint8))
        assert not torch.equal(got, want)


def np_tables(n, D):
    a = np.arange(n)[:, None] * 10000.0 ** (-2.0 * np.arange(D // 2) / D)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


@pytest.mark.parametrize("fmt", FMTS)
def test_offsets_past_32_bits(fmt):
    """Pools whose byte offsets (and, in bf16, element offsets) pass 2^32: the pages at the far end."""
    page, hkv, D, hq = 64, 8, 128, 16
    row = D * 2 if fmt == "bf16" else D // 2
    pages = (5 << 30) // (page * hkv * row) if fmt == "mx" else (9 << 30) // (page * hkv * row)
    cache = S.alloc_kv_cache(pages, page, hkv, D, fmt, DEV)
    assert cache.k.numel() * cache.k.element_size() > 1 << 32
    lens, per = [300, 70], [300, 3]
    near = np.arange(pages - 7, pages).astype(np.int32)
    table = np.stack([near[:5], np.array([near[5], near[6], 0, 0, 0], np.int32)])
    offsets = np.array([0, 300, 370], np.int32)
    rng = np.random.default_rng(0)
    x = R.bf16(rng.standard_normal((370, 2 * hkv * D)))
    t = [torch.from_numpy(a).to(DEV) for a in (offsets, np.array([300, 70], np.int32), table)]
    S.sharq_kv_append(None, x[:, :hkv * D].to(DEV), x[:, hkv * D:].to(DEV), cache, S.KVBatch(*t, 370, 300, 300))
    k, v = S.sharq_kv_read(cache, S.KVBatch(*t, 370, 300, 300))
    if fmt == "bf16":
        assert torch.equal(k.cpu(), x[:, :hkv * D]) and torch.equal(v.cpu(), x[:, hkv * D:])
    # the same pages at the front of a small pool
    small = S.KVCache(fmt, *(None if p is None else p[-7:].clone() for p in
                             (cache.k, cache.v, cache.k_scale, cache.v_scale)))
    q = R.bf16(rng.standard_normal((370, hq * D))).to(DEV)
    for per, rows in (([300, 70], 370), ([1, 3], 4)):
        o = torch.tensor(np.concatenate([[0], np.cumsum(per)]), dtype=torch.int32, device=DEV)
        far = S.KVBatch(o, t[1], t[2], rows, max(per), 300)
        low = S.KVBatch(o, t[1], t[2] - (pages - 7), rows, max(per), 300)
        assert torch.equal(S.sharq_attention(q[:rows], cache, far), S.sharq_attention(q[:rows], small, low))


@pytest.mark.parametrize("fmt", FMTS)
def test_a_sequence_served_step_by_step(fmt):
    """A prompt in chunks and then single tokens through append and attention, as a program serves it, against the whole
    prompt in one call: the same keys are read, so the outputs agree to the roundings of two calls."""
    hq, hkv, D, page, n = 8, 2, 128, 16, 150
    rng = np.random.default_rng(9)
    x = R.bf16(rng.standard_normal((n, (hq + 2 * hkv) * D))).to(DEV)
    cos, sin = (torch.from_numpy(t).to(DEV) for t in np_tables(n, D))
    table = torch.randperm(12, generator=torch.Generator().manual_seed(1)).to(torch.int32)[None].to(DEV)
    cache = S.alloc_kv_cache(12, page, hkv, D, fmt, DEV)
    w = hq * D, (hq + hkv) * D
    got, lses = [], []
    at = 0
    for m in [64, 33, 20] + [1] * 33:
        batch = S.KVBatch(torch.tensor([0, m], dtype=torch.int32, device=DEV),
                          torch.tensor([at + m], dtype=torch.int32, device=DEV), table, m, m, 12 * page)
        y = x[at:at + m]
        q = S.sharq_kv_append(y[:, :w[0]], y[:, w[0]:w[1]], y[:, w[1]:], cache, batch, cos, sin)
        lse = torch.empty((m, hq), device=DEV)
        got.append(S.sharq_attention(q, cache, batch, lse=lse))
        lses.append(lse)
        at += m
    offsets, lens = [0, n], [n]
    whole = S.KVBatch(torch.tensor(offsets, dtype=torch.int32, device=DEV),
                      torch.tensor(lens, dtype=torch.int32, device=DEV), table, n, n, 12 * page)
    q = S.sharq_kv_append(x[:, :w[0]], x[:, w[0]:w[1]], x[:, w[1]:], cache, whole, cos, sin)
    check(q, cache, whole, offsets, lens, table.cpu().numpy(), torch.cat(got), torch.cat(lses))
    lse = torch.empty((n, hq), device=DEV)
    check(q, cache, whole, offsets, lens, table.cpu().numpy(), S.sharq_attention(q, cache, whole, lse=lse), lse)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("seqs,new,length", [(1, 130, 130), (5, 1, 300)])
def test_between_the_linears_of_a_layer(seqs, new, length, fmt):
    """qkv linear, append, attention and the o projection's preparation, each on the output of the one before: the
    append on slices of the linear's output, the attention against the definition on what was appended, and the
    preparation byte by byte as on a copy of the attention's output."""
    hq, hkv, D, page, H = 8, 2, 64, 16, 256
    rng = np.random.default_rng(seqs)
    batch, offsets, lens, table, pages = make_batch([new] * seqs, [length] * seqs, page)
    cache = filled_cache(pages, page, hkv, D, fmt)
    rows = batch.rows
    h = R.bf16(rng.standard_normal((rows, H))).to(DEV)
    w = S.sharq_quantize_weight(R.bf16(rng.standard_normal(((hq + 2 * hkv) * D, H)) * 0.05).to(DEV))
    gamma = R.bf16(1 + 0.1 * rng.standard_normal(H)).to(DEV)
    cos, sin = np_tables(length, D)
    act, z = S.sharq_prepare_linear(h, gamma, w, 1e-5)
    qw, kw = hq * D, (hq + hkv) * D
    q = S.sharq_kv_append(z[:, :qw], z[:, qw:kw], z[:, kw:], cache, batch, torch.from_numpy(cos).to(DEV),
                          torch.from_numpy(sin).to(DEV))
    lse = torch.empty((rows, hq), device=DEV)
    a = S.sharq_attention(q, cache, batch, lse=lse)
    p = S.sharq_prepare(a, None)
    p2 = S.sharq_prepare(a.clone(), None)
    torch.cuda.synchronize()
    zs = z.float().cpu().numpy().reshape(rows, -1, D)
    seq, pos = R.positions(offsets, lens, rows)
    y = R.rotate32(zs[:, :hq + hkv], cos[pos], sin[pos])
    assert np.array_equal(q.float().cpu().numpy(), R.bf16(y[:, :hq].reshape(rows, -1)).float().numpy())
    k, v = S.sharq_kv_read(cache, batch)
    for got, src in ((k, y[:, hq:]), (v, zs[:, hq + hkv:])):
        val = R.bf16(src).double().numpy() if fmt == "bf16" else R.mx_values(*R.mx_quantize(src))
        assert np.array_equal(got.double().cpu().numpy(), val.reshape(rows, -1))
    check(q, cache, batch, offsets, lens, table, a, lse)
    for name in ("sp_codes", "sp_meta", "sp_scale", "dn_codes", "dn_scale"):
        assert torch.equal(getattr(p, name), getattr(p2, name))


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("per,lens", [([1, 2], [40, 20]), ([60], [60])])
def test_pool_without_pages(per, lens, fmt):
    batch, offsets, ln, table, pages = make_batch(per, lens, 16)
    cache = S.alloc_kv_cache(0, 16, 2, 128, fmt, DEV)
    x = torch.randn((batch.rows, 256), device=DEV).to(torch.bfloat16)
    assert torch.equal(S.sharq_kv_append(x, x, x, cache, batch), x)
    k, v = S.sharq_kv_read(cache, batch)
    assert not k.any() and not v.any()
    lse = torch.zeros((batch.rows, 2), device=DEV)
    out = S.sharq_attention(x, cache, batch, lse=lse)
    assert not out.any() and torch.isneginf(lse).all()
