"""The paged key/value cache without a GPU: the cache's indexing and the tiles
that attention walks (csrc/sharq_kv.hpp, compiled for the host), the refusals of
the C ABI and of the binding, and the reference that the GPU tests compare with."""

import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import kv_ref as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2606_26587_amd", "libsharq.so")

SHIM = r"""
#include "sharq_kv.hpp"
using namespace sharq;
extern "C" {
int row(int page, int t, int pages, int heads, int head, int shift) { return kv_row(page, t, pages, heads, head, shift); }
// tiles of a span: their first tokens into `start`; returns how many; {low, hi} into `range`
int span(int t0, int t1, int p_lo, int p_hi, int window, int sinks, int T, int* start, int* range, int most) {
  const KvSpan s = kv_span(t0, t1, p_lo, p_hi, window, sinks, T);
  range[0] = s.low, range[1] = s.hi;
  for (int i = 0; i < s.n && i < most; ++i) start[i] = kv_tile_start(s, t0, i, T);
  return s.n;
}
// {few, shared, own tiles, chunks, tiles of a chunk, prefix ..., slots}; workspace bytes
int64_t plan(int64_t seqs, int64_t rows, int64_t max_rows, int64_t max_len, int heads, int group, int D, int mx,
             int64_t window, int64_t sinks, int64_t prefix, int64_t* out) {
  const AttnPlan p = attn_plan(seqs, rows, max_rows, max_len, heads, group, D, mx, window, sinks, prefix);
  const int64_t v[] = {p.few, p.shared, p.own.tiles, p.own.chunks, p.own.chunk_tiles, p.prefix.tiles, p.prefix.chunks,
                       p.prefix.chunk_tiles, p.slots};
  for (int i = 0; i < 9; ++i) out[i] = v[i];
  return attn_workspace(rows * heads * group, p.slots, D);
}
int mixed(int64_t seqs, int64_t rows, int64_t max_rows, int64_t max_len, int heads, int group, int D, int mx,
          int64_t window, int64_t sinks, int64_t prefix) {
  const AttnPlan p = attn_plan(seqs, rows, max_rows, max_len, heads, group, D, mx, window, sinks, prefix);
  return p.mixed ? 1 + (p.few || p.shared || p.slots) : 0;   // 2: a plan that may not be
}
int tile_rows() { return kAttnRows; }
int tile_tokens() { return kAttnTile; }
}
"""


@pytest.fixture(scope="module")
def kv(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv")
    (d / "shim.cpp").write_text(SHIM)
    so = str(d / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-shared", "-fPIC",
                    "-I", os.path.join(ROOT, "paper_2606_26587_amd", "csrc"), str(d / "shim.cpp"), "-o", so],
                   check=True)
    return ctypes.CDLL(so)


def test_rows_of_pages_inside_and_outside_the_pool(kv):
    pages, heads, shift = 5, 3, 4
    seen = set()
    for page in (-2 ** 31, -1, 0, 4, 5, 2 ** 31 - 1):
        for head in range(heads):
            for t in list(range(16)) + [2 ** 30 - 1]:
                r = kv.row(page, t, pages, heads, head, shift)
                if not 0 <= page < pages:
                    assert r == -1
                else:
                    assert r == (page * heads + head) * 16 + t % 16
                    assert 0 <= r < pages * heads * 16
                    seen.add(r)
    assert len(seen) == 2 * heads * 16
    # the largest pool whose rows are counted in 32 bits
    assert kv.row(2 ** 21 - 2, 1023, 2 ** 21 - 1, 1, 0, 10) == 2 ** 31 - 1024 - 1


@pytest.mark.parametrize("T", [32, 64])
def test_spans_cover_what_is_seen_once(kv, T):
    rng = np.random.default_rng(T)
    start, rg = (ctypes.c_int * 4096)(), (ctypes.c_int * 2)()
    big = 2 ** 31 - 1
    for _ in range(3000):
        length = int(rng.integers(0, 900))
        n = int(rng.integers(1, 80))
        p_lo = length - n
        p_hi = p_lo + int(rng.integers(0, n))
        window = int(rng.choice([1, 2, T - 1, T, T + 1, 200, big, int(rng.integers(1, 1000))]))
        sinks = int(rng.choice([0, 0, 1, 4, T, T + 1, 300, big]))
        t0 = int(rng.choice([0, 0, 16, 48, 128, 512]))
        count = kv.span(t0, length, p_lo, p_hi, window, sinks, T, start, rg, 4096)
        assert count <= 4096
        tiles = list(start[:count])
        assert tiles == sorted(set(tiles)) and all((t - t0) % T == 0 and t >= t0 for t in tiles)
        t = np.arange(t0, max(length, t0))
        p = np.arange(p_lo, p_hi + 1)[:, None]
        sees = ((t <= p) & ((p - t < window) | (t < sinks))).any(0)
        covered = np.zeros(len(t) + T, bool)
        for x in tiles:
            covered[x - t0:x - t0 + T] = True
            # no tile is walked for nothing, but for one that lies between what two rows see
            assert x < rg[1]
        assert covered[:len(t)][sees].all()
        mine = (t < rg[1]) & ((t >= rg[0]) | (t < sinks))
        assert (mine[sees]).all()               # what some row sees is loaded
        full = (p_hi - p_lo) < window           # (rows further apart than the window leave gaps)
        assert not full or (mine == sees).all()


def test_span_at_the_ends_of_the_range(kv):
    start, rg = (ctypes.c_int * 4)(), (ctypes.c_int * 2)()
    big = 2 ** 31 - 1
    assert kv.span(0, 2 ** 30, 2 ** 30 - 1, 2 ** 30 - 1, big, 0, 64, start, rg, 4) == 2 ** 24
    assert kv.span(0, 2 ** 30, 2 ** 30 - 1, 2 ** 30 - 1, 1, 0, 64, start, rg, 4) == 1 and start[0] == 2 ** 30 - 64
    assert kv.span(0, 0, -5, -1, 1, 7, 64, start, rg, 4) == 0
    assert kv.span(0, 5, -2 ** 31 + 8, -1, big, big, 64, start, rg, 4) == 0


def test_plans_cover_every_tile_of_every_row(kv):
    """Whatever the sequences within the batch's bounds, the plan's workgroups take all tiles of tokens that any tile of
    rows sees, have a tile of rows each, and fit the workspace."""
    kv.plan.restype = ctypes.c_int64
    kv.plan.argtypes = [ctypes.c_int64] * 4 + [ctypes.c_int] * 4 + [ctypes.c_int64] * 3 + [ctypes.POINTER(ctypes.c_int64)]
    R, T = kv.tile_rows(), kv.tile_tokens()
    rng = np.random.default_rng(11)
    start, rg, out = (ctypes.c_int * 1)(), (ctypes.c_int * 2)(), (ctypes.c_int64 * 9)()
    big = 2 ** 31 - 1

    def tiles(t0, length, p_lo, p_hi, window, sinks, tok):
        return kv.span(t0, length, p_lo, p_hi, window, sinks, tok, start, rg, 0)

    kinds = set()
    for _ in range(1500):
        seqs = int(rng.integers(1, 40))
        most = int(rng.choice([1, 2, 4, 9, 40, 300, 2000]))
        n = rng.integers(0, most + 1, seqs)
        n[int(rng.integers(seqs))] = most
        lens = np.maximum(n + rng.integers(0, int(rng.choice([2, 100, 5000])), seqs), 0)
        max_len = int(lens.max()) + int(rng.choice([0, 0, 17, 3000]))
        rows = int(n.sum()) + int(rng.integers(0, 5))
        max_rows = most + int(rng.choice([0, 0, 3, 100]))
        heads, group = [(8, 4), (4, 7), (1, 1), (2, 16), (1, 128), (4, 8), (3, 3)][int(rng.integers(7))]
        D, mx = int(rng.choice([64, 128])), int(rng.integers(2))
        window = int(rng.choice([big, big, 1, 16, 100, 1000]))
        sinks = int(rng.choice([0, 1, 4, 64, 300, big]))
        prefix = int(rng.choice([0, 0, 16, 256, 1024]))
        prefix = prefix if prefix <= max_len else 0
        size = kv.plan(seqs, rows, max_rows, max_len, heads, group, D, mx, window, sinks, prefix, out)
        few, shared, own_tiles, own_chunks, own_each, pre_tiles, pre_chunks, pre_each, slots = out
        kinds.add((few, shared, slots > 0))
        assert own_chunks >= 1 and own_each >= 1 and own_chunks * own_tiles * heads < 2 ** 23
        assert slots == (own_chunks + pre_chunks if shared else own_chunks if own_chunks > 1 else 0)
        assert size == (0 if slots == 0 else -(-rows * heads * group * slots * 8 // 16) * 16
                        + rows * heads * group * slots * D * 4)
        t0 = prefix if shared else 0
        used = 0
        for i in range(seqs):
            base = int(lens[i] - n[i])
            if few:
                assert n[i] * group <= 16 * few
                if n[i]:
                    tok = 64 if mx else 32
                    assert tiles(t0, int(lens[i]), base, int(lens[i]) - 1, window, sinks, tok) <= own_chunks * own_each
                continue
            all_rows = int(n[i]) * group
            for r0 in range(0, all_rows, R):
                last = min(all_rows, r0 + R) - 1
                used += 1
                got = tiles(t0, int(lens[i]), base + r0 // group, base + last // group, window, sinks, T)
                assert got <= own_chunks * own_each
        assert few or used <= own_tiles
        if shared:
            assert window >= max_len and pre_tiles * R >= int(n.sum()) * group
            assert -(-prefix // T) <= pre_chunks * pre_each
    assert {k[0] for k in kinds} == {0, 1, 2, 4} and {k[1:] for k in kinds} == {(0, False), (0, True), (1, True)}


def test_mixed_plans(kv):
    """Both kernels in one launch: unsplit batches of some long and many short sequences on an MXFP4 cache, no others."""
    kv.mixed.argtypes = [ctypes.c_int64] * 4 + [ctypes.c_int] * 4 + [ctypes.c_int64] * 3
    big = 2 ** 31 - 1
    assert kv.mixed(64, 2063, 2000, 4000, 8, 4, 128, 1, big, 0, 0) == 1
    assert kv.mixed(64, 2063, 2000, 4000, 8, 4, 128, 1, 100, 4, 1024) == 1      # a window: the prefix is like any page
    assert kv.mixed(64, 2063, 2000, 4000, 8, 4, 128, 0, big, 0, 0) == 0         # bf16
    assert kv.mixed(64, 2063, 2000, 4000, 8, 4, 128, 1, big, 0, 1024) == 0      # a shared prefix
    assert kv.mixed(64, 100000, 2000, 4000, 8, 4, 128, 1, big, 0, 0) == 0       # of about the same lengths
    assert kv.mixed(64, 64, 1, 4000, 8, 4, 128, 1, big, 0, 0) == 0              # few rows all
    assert kv.mixed(2, 2001, 2000, 4000, 1, 4, 128, 1, big, 0, 0) == 0          # split
    rng = np.random.default_rng(5)
    for _ in range(3000):
        seqs, most = int(rng.integers(1, 3000)), int(rng.integers(1, 5000))
        got = kv.mixed(seqs, int(rng.integers(most, seqs * most + 1)), most, most + int(rng.integers(0, 9000)),
                       int(rng.integers(1, 17)), int(rng.integers(1, 33)), int(rng.choice([64, 128])),
                       int(rng.integers(2)), int(rng.choice([big, 50])), int(rng.integers(0, 9)), 0)
        assert got in (0, 1)


# ---------------------------------------------------------------------------
# C ABI
# ---------------------------------------------------------------------------

OK, EINVAL, EUNSUPPORTED, EALIGN = 0, 1, 2, 3
FAKE = 1 << 20   # never dereferenced: every call below is refused (or empty) before any launch


class Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("fmt", ctypes.c_int), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p), ("scale_rule", ctypes.c_int)]


class Batch(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int64), ("rows", ctypes.c_int64), ("max_rows", ctypes.c_int64),
                ("max_len", ctypes.c_int64), ("ld_table", ctypes.c_int64), ("row_offsets", ctypes.c_void_p),
                ("lens", ctypes.c_void_p), ("page_table", ctypes.c_void_p)]


class Attn(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("window", ctypes.c_int64), ("sinks", ctypes.c_int64),
                ("prefix_table", ctypes.c_void_p), ("prefix_len", ctypes.c_int64)]


def cache(**kw):
    d = dict(pages=8, page_size=16, kv_heads=2, head_dim=128, fmt=0, k=FAKE, v=FAKE, k_scale=None, v_scale=None,
             scale_rule=0)
    d.update(kw)
    return Cache(**d)


def batch(**kw):
    d = dict(seqs=2, rows=4, max_rows=2, max_len=64, ld_table=4, row_offsets=FAKE, lens=FAKE, page_table=FAKE)
    d.update(kw)
    return Batch(**d)


def attn(**kw):
    d = dict(scale=0.1, window=0, sinks=0, prefix_table=None, prefix_len=0)
    d.update(kw)
    return Attn(**d)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(LIB):
        pytest.skip("libsharq.so not built")
    lib = ctypes.CDLL(LIB)
    i64, vp, p = ctypes.c_int64, ctypes.c_void_p, ctypes.POINTER
    lib.sharq_kv_buffer_bytes.restype = lib.sharq_attention_workspace_bytes.restype = ctypes.c_size_t
    lib.sharq_kv_buffer_bytes.argtypes = [p(Cache), ctypes.c_int32]
    lib.sharq_kv_append.argtypes = [vp, vp, vp, ctypes.c_int, i64, i64, i64, i64, vp, vp, i64, vp, p(Cache), p(Batch),
                                    vp, i64, vp]
    lib.sharq_kv_read.argtypes = [p(Cache), p(Batch), vp, i64, vp, i64, ctypes.c_int, vp]
    lib.sharq_attention_workspace_bytes.argtypes = [p(Cache), p(Batch), p(Attn), i64]
    lib.sharq_attention.argtypes = [vp, ctypes.c_int, i64, i64, p(Cache), p(Batch), p(Attn), vp, i64, vp, vp,
                                    ctypes.c_size_t, vp]
    return lib


def append(L, c=None, b=None, q=FAKE, k=FAKE, v=FAKE, dt=0, heads=4, ldq=512, ldk=256, ldv=256, cos=FAKE, sin=FAKE,
           angles=64, pos=None, out=FAKE, ldo=512):
    return L.sharq_kv_append(q, k, v, dt, heads, ldq, ldk, ldv, cos, sin, angles, pos,
                             ctypes.byref(c or cache()), ctypes.byref(b or batch()), out, ldo, None)


def read(L, c=None, b=None, k=FAKE, v=FAKE, ldk=256, ldv=256, dt=0):
    return L.sharq_kv_read(ctypes.byref(c or cache()), ctypes.byref(b or batch()), k, ldk, v, ldv, dt, None)


def attention(L, c=None, b=None, t=None, q=FAKE, dt=0, heads=4, ldq=512, o=FAKE, ldo=512, lse=None, ws=FAKE,
              size=1 << 40):
    return L.sharq_attention(q, dt, heads, ldq, ctypes.byref(c or cache()), ctypes.byref(b or batch()),
                             ctypes.byref(t or attn()), o, ldo, lse, ws, size, None)


BAD_CACHES = [
    (dict(pages=-1), EINVAL), (dict(page_size=0), EINVAL), (dict(page_size=24), EINVAL), (dict(page_size=-16), EINVAL),
    (dict(page_size=8), EUNSUPPORTED), (dict(page_size=2048), EUNSUPPORTED), (dict(kv_heads=0), EINVAL),
    (dict(head_dim=96), EUNSUPPORTED), (dict(head_dim=0), EINVAL), (dict(fmt=2), EINVAL), (dict(scale_rule=2), EINVAL),
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k=FAKE + 8), EALIGN), (dict(fmt=1), EINVAL),
    (dict(fmt=1, k_scale=FAKE, v_scale=FAKE + 2), EALIGN), (dict(pages=1 << 26), EUNSUPPORTED),
]
BAD_BATCHES = [
    (dict(seqs=-1), EINVAL), (dict(rows=-1), EINVAL), (dict(rows=1 << 31), EINVAL), (dict(max_rows=-1), EINVAL),
    (dict(max_len=-1), EINVAL), (dict(ld_table=3), EINVAL), (dict(ld_table=-1), EINVAL),
    (dict(row_offsets=None), EINVAL), (dict(lens=None), EINVAL), (dict(page_table=None), EINVAL),
    (dict(lens=FAKE + 2), EALIGN), (dict(seqs=1 << 17), EUNSUPPORTED), (dict(max_len=1 << 31, ld_table=1 << 30), EUNSUPPORTED),
]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_bad_caches_are_refused(L, bad, status):
    for call in (append, read, attention):
        assert call(L, c=cache(**bad)) == status


@pytest.mark.parametrize("bad,status", BAD_BATCHES)
def test_bad_batches_are_refused(L, bad, status):
    for call in (append, read, attention):
        assert call(L, b=batch(**bad)) == status


def test_bad_append_arguments(L):
    for kw, status in [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL),
                       (dict(cos=None), EINVAL), (dict(sin=None), EINVAL), (dict(angles=-1), EINVAL),
                       (dict(cos=None, sin=None, pos=FAKE), EINVAL), (dict(heads=-1), EINVAL), (dict(ldq=511), EINVAL),
                       (dict(ldk=255), EINVAL), (dict(ldv=255), EINVAL), (dict(ldo=511), EINVAL), (dict(dt=1), EUNSUPPORTED),
                       (dict(ldq=513), EALIGN), (dict(ldk=260), EALIGN), (dict(k=FAKE + 2), EALIGN),
                       (dict(cos=FAKE + 4), EALIGN), (dict(pos=FAKE + 1), EALIGN), (dict(heads=2000, ldq=1 << 20, ldo=1 << 20), EUNSUPPORTED),
                       (dict(b=batch(rows=1 << 25)), EUNSUPPORTED)]:
        assert append(L, **kw) == status, kw


def test_bad_read_arguments(L):
    for kw, status in [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(ldk=255), EINVAL), (dict(dt=2), EUNSUPPORTED),
                       (dict(ldv=260), EALIGN), (dict(v=FAKE + 8), EALIGN)]:
        assert read(L, **kw) == status, kw


def test_bad_attention_arguments(L):
    nan, inf = float("nan"), float("inf")
    for kw, status in [(dict(q=None), EINVAL), (dict(o=None), EINVAL), (dict(heads=0), EINVAL), (dict(heads=3), EINVAL),
                       (dict(heads=258, ldq=1 << 20, ldo=1 << 20), EUNSUPPORTED), (dict(ldq=511), EINVAL),
                       (dict(ldo=511), EINVAL), (dict(dt=1), EUNSUPPORTED), (dict(ldo=516), EALIGN),
                       (dict(q=FAKE + 4), EALIGN), (dict(lse=FAKE + 2), EALIGN), (dict(ws=FAKE + 8), EALIGN),
                       (dict(t=attn(scale=0.0)), EINVAL), (dict(t=attn(scale=-1.0)), EINVAL),
                       (dict(t=attn(scale=nan)), EINVAL), (dict(t=attn(scale=inf)), EINVAL),
                       (dict(t=attn(window=-1)), EINVAL), (dict(t=attn(sinks=-1)), EINVAL),
                       (dict(t=attn(prefix_len=16)), EINVAL), (dict(t=attn(prefix_len=8, prefix_table=FAKE)), EINVAL),
                       (dict(t=attn(prefix_len=-16, prefix_table=FAKE)), EINVAL),
                       (dict(t=attn(prefix_len=80, prefix_table=FAKE)), EINVAL),
                       (dict(t=attn(prefix_len=16, prefix_table=FAKE + 2)), EALIGN),
                       (dict(b=batch(rows=1 << 25)), EUNSUPPORTED)]:
        assert attention(L, **kw) == status, kw


def test_scales_out_of_range(L):
    """A scale whose product with log2 e, or with the running maximum's start, is no normal fp32 number."""
    for scale in (1e-45, 2.0 ** -126, 1.5e-38, 2.0 ** -101, 2.0 ** 101, 3e38):
        assert attention(L, t=attn(scale=scale)) == EUNSUPPORTED, scale
        assert L.sharq_attention_workspace_bytes(ctypes.byref(cache()), ctypes.byref(batch(max_len=4096, ld_table=256)),
                                                 ctypes.byref(attn(scale=scale)), 4) == 0


def test_attention_in_place_is_refused(L):
    assert attention(L, q=FAKE, o=FAKE, ws=FAKE, size=1 << 30) == EINVAL


def test_empty_calls_do_nothing(L):
    for b in (batch(seqs=0), batch(rows=0), batch(seqs=0, rows=0, ld_table=0, row_offsets=None, lens=None, page_table=None)):
        assert append(L, b=b, q=None, k=None, v=None, out=None) == OK
        assert read(L, b=b, k=None, v=None) == OK
        assert attention(L, b=b, q=None, o=None, ws=None, size=0) == OK
    assert attention(L, b=batch(max_rows=0), q=None, o=None, ws=None, size=0) == OK


def test_padding_rows_take_no_workspace(L):
    """Only rows that sequences can own (seqs times max_rows) have partial results."""
    def size(c=cache(), heads=4, **kw):
        return L.sharq_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(batch(max_len=4096, ld_table=256, **kw)),
                                                 ctypes.byref(attn()), heads)
    for seqs, max_rows in ((1, 1), (3, 1), (2, 8), (1, 300)):
        want = size(seqs=seqs, rows=seqs * max_rows, max_rows=max_rows)
        assert want > 0
        for rows in (seqs * max_rows + 1, 5000, 1 << 20):
            assert size(seqs=seqs, rows=rows, max_rows=max_rows) == want
        assert size(seqs=seqs, rows=seqs * max_rows, max_rows=1 << 40) == size(seqs=seqs, rows=seqs * max_rows,
                                                                               max_rows=seqs * max_rows)


def test_null_structs(L):
    c, b, t = cache(), batch(), attn()
    r = ctypes.byref
    assert L.sharq_kv_read(None, r(b), FAKE, 256, FAKE, 256, 0, None) == EINVAL
    assert L.sharq_kv_read(r(c), None, FAKE, 256, FAKE, 256, 0, None) == EINVAL
    assert L.sharq_attention(FAKE, 0, 4, 512, r(c), r(b), None, FAKE, 512, None, None, 0, None) == EINVAL
    assert L.sharq_attention_workspace_bytes(None, r(b), r(t), 4) == 0
    assert L.sharq_kv_buffer_bytes(None, 0) == 0


def test_buffer_bytes(L):
    size = lambda c: [L.sharq_kv_buffer_bytes(ctypes.byref(c), i) for i in range(-1, 5)]  # noqa: E731
    n = 8 * 16 * 2 * 128
    assert size(cache(k=None, v=None)) == [0, n * 2, n * 2, 0, 0, 0]
    assert size(cache(fmt=1)) == [0, n // 2, n // 2, n // 32, n // 32, 0]
    assert size(cache(page_size=17)) == [0] * 6


# ---------------------------------------------------------------------------
# Binding
# ---------------------------------------------------------------------------

def test_binding_refuses_wrong_tensors(monkeypatch):
    from paper_2606_26587_amd import sharq as S

    class NoLaunch:
        sharq_status_str = S.lib.sharq_status_str

        def __getattr__(self, name):
            raise AssertionError(f"{name} was called")

    real = S.lib
    c = S.alloc_kv_cache(4, 16, 2, 128, "bf16", "cpu")
    m = S.alloc_kv_cache(4, 16, 2, 64, "mx", "cpu")
    assert (c.pages, c.kv_heads, c.page_size, c.head_dim) == (4, 2, 16, 128)
    assert (m.pages, m.kv_heads, m.page_size, m.head_dim) == (4, 2, 16, 64)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    b = S.KVBatch(i32(0, 1, 2), i32(5, 6), torch.zeros(2, 1, dtype=torch.int32), 2, 1, 16)
    q, k = torch.zeros(2, 512, dtype=torch.bfloat16), torch.zeros(2, 256, dtype=torch.bfloat16)

    def refused(f, *a, **kw):
        with pytest.raises(S.SharqError) as e:
            f(*a, **kw)
        assert e.value.status == S.EINVAL

    refused(S.sharq_attention, q, c, b)                  # buffers that are not on a GPU
    refused(S.sharq_kv_append, q, k, k, c, b)
    refused(S.sharq_kv_read, c, b)
    monkeypatch.setattr(S, "_here", lambda *a: None)
    monkeypatch.setattr(S, "lib", NoLaunch())
    refused(S.KVCache, "bf16", c.k.half(), c.v)
    refused(S.KVCache, "bf16", c.k, c.v[:2])
    refused(S.KVCache, "bf16", c.k.transpose(1, 2), c.v.transpose(1, 2))
    refused(S.KVCache, "mx", m.k, m.v)
    refused(S.KVCache, "mx", m.k, m.v, m.k_scale, m.v_scale[..., :1])
    refused(S.KVBatch, i32(0, 1), i32(5, 6), torch.zeros(2, 1, dtype=torch.int32), 2, 1, 16)
    refused(S.KVBatch, i32(0, 1, 2), i32(5, 6).long(), torch.zeros(2, 1, dtype=torch.int32), 2, 1, 16)
    refused(S.KVBatch, i32(0, 1, 2), i32(5, 6), torch.zeros(1, 4, dtype=torch.int32), 2, 1, 16)
    refused(S.KVBatch, i32(0, 1, 2), i32(5, 6), torch.zeros(4, 2, dtype=torch.int32).T, 2, 1, 16)
    refused(S.sharq_attention, q.float(), c, b)
    refused(S.sharq_attention, q[:1], c, b)
    refused(S.sharq_attention, q[:, :500], c, b)
    refused(S.sharq_attention, q, c, b, out=k)
    refused(S.sharq_attention, q, c, b, lse=torch.zeros(2, 2))
    refused(S.sharq_attention, q, c, b, prefix_table=i32(0), prefix_len=32)
    refused(S.sharq_attention, torch.zeros(512, 2, dtype=torch.bfloat16).T, c, b)
    refused(S.sharq_kv_append, q, k, q, c, b)
    refused(S.sharq_kv_append, q, k, k, c, b, q_out=k)
    refused(S.sharq_kv_append, q, k, k, c, b, cos=torch.zeros(9, 32), sin=torch.zeros(9, 32))
    refused(S.sharq_kv_append, q, k, k, c, b, cos=torch.zeros(9, 64))
    refused(S.sharq_kv_append, q, k, k, c, b, cos=torch.zeros(9, 64), sin=torch.zeros(9, 64), positions=i32(1))
    refused(S.sharq_kv_read, c, b, k_out=q)
    # what the library itself refuses: a negative scale, a sequence longer than its page table
    monkeypatch.setattr(S, "lib", real)
    stream = type("Stream", (), {"cuda_stream": 0})
    refused(S.sharq_attention, q, c, b, scale=-1.0, workspace=torch.zeros(16), stream=stream)
    long = S.KVBatch(i32(0, 1, 2), i32(5, 6), torch.zeros(2, 1, dtype=torch.int32), 2, 1, 17)
    refused(S.sharq_kv_read, c, long, stream=stream)


# ---------------------------------------------------------------------------
# The reference itself
# ---------------------------------------------------------------------------

def test_reference_attention_is_softmax_over_the_visible_tokens():
    rng = np.random.default_rng(0)
    pages, hkv, ps, D = 6, 2, 4, 8
    kp, vp = rng.standard_normal((2, pages, hkv, ps, D))
    table = np.array([[3, 0, 5], [1, 4, 2]])
    q = rng.standard_normal((5, 4, D))
    offsets, lens = [0, 3, 4], [10, 7]
    o, lse, mag, _ = R.attention(q, kp, vp, offsets, lens, table, 0.3, window=3, sinks=1)
    for i, (s, p) in enumerate([(0, 7), (0, 8), (0, 9), (1, 6)]):
        k = np.concatenate([kp[x] for x in table[s]], 1)
        v = np.concatenate([vp[x] for x in table[s]], 1)
        t = np.arange(12)
        for h in range(4):
            z = np.where((t <= p) & ((t > p - 3) | (t < 1)), 0.3 * k[h // 2] @ q[i, h], -np.inf)
            w = np.exp(z) / np.exp(z).sum()
            assert np.allclose(o[i, h], w @ v[h // 2]) and np.allclose(lse[i, h], np.log(np.exp(z).sum()))
            assert np.allclose(mag[i, h], w @ np.abs(v[h // 2]))
    assert np.isnan(o[4]).all()


@pytest.mark.parametrize("rule", ["floor", "ceil"])
def test_reference_quantizer_agrees_with_the_oracle(rule):
    from oracle import sharq_oracle as O
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((7, 128)) * np.exp2(rng.integers(-20, 20, (7, 1)))).astype(np.float32)
    codes, scales = R.mx_quantize(x, rule)
    v = R.mx_values(codes, scales)
    grid = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
    unit = np.exp2(scales.astype(float) - 127).repeat(32, -1)
    near = grid[np.abs(np.abs(x / unit)[..., None] - grid).argmin(-1)]
    assert np.allclose(np.abs(v), near * unit)
    peak = np.abs(x).reshape(7, 4, 32).max(-1)
    e = np.floor(np.log2(peak)) - 2 if rule == "floor" else np.ceil(np.log2(peak / 6))
    assert np.array_equal(e, scales.astype(float) - 127)
    c2, _, s2, deq = O.mx_quantize(x, None, rule)
    assert np.array_equal(np.asarray(s2).reshape(scales.shape), scales) and np.array_equal(deq, v)
