"""The 8-bit key/value cache without a GPU: the reference itself, sizes, refusals of the C ABI and of the binding, and
the launches' work split."""

import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import kv8_ref as K
from test_kv_cpu import EALIGN, EINVAL, FAKE, L, OK, ROOT, append, attention, batch, cache, kv, read  # noqa: F401


def f8(**kw):
    return cache(**{**dict(fmt=2, k_scale=FAKE, v_scale=FAKE), **kw})


def test_codes_are_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, K.VALUES, equal_nan=True)
    x = np.concatenate([np.linspace(-460, 460, 40001), np.exp2(np.linspace(-13, 9, 5000)), K.VALUES[:0x7F],
                        (K.VALUES[:0x7E] + K.VALUES[1:0x7F]) / 2])
    x = x.astype(np.float32)
    want = torch.from_numpy(np.clip(x, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(K.encode(x), want)
    assert list(K.encode([np.nan, np.inf, -np.inf, -0.0])) == [0x7F, 0x7F, 0x7F, 0x80]


def test_exponents():
    for rule, peak, want in [("floor", 448.0, 0), ("floor", 511.0, 0), ("floor", 512.0, 1), ("ceil", 448.0, 0),
                             ("ceil", 448.1, 1), ("ceil", 256.0, 0), ("ceil", 224.0, -1), ("ceil", 225.0, 0),
                             ("floor", 0.0, -117), ("ceil", 1e-40, -117), ("floor", 3.3e38, 119)]:
        assert K.exponent(peak, rule) == want, (rule, peak)
    rng = np.random.default_rng(0)
    x = rng.standard_normal((2, 3, 32, 64)) * np.exp2(rng.integers(-30, 30, (2, 3, 32, 1)))
    c, e = K.quantize(x, "ceil")
    assert (np.abs(K.VALUES[c]) <= 448).all() and np.abs(K.VALUES[c]).reshape(2, 3, 2, -1).max(-1).min() > 223
    v = K.values(c, e)
    unit = np.exp2(e.astype(float) - 127).repeat(16, -1)[..., None]
    # half a step of a value, or half of the least code
    assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, unit * 2.0 ** -10)).all()


def test_the_least_values_are_normal_bf16():
    v = K.VALUES[1:0x7F] * 2.0 ** K.LEAST
    assert v.min() == 2.0 ** -126
    assert np.array_equal(torch.from_numpy(v).to(torch.bfloat16).double().numpy(), v)


def test_sizes(L):  # noqa: F811
    size = lambda c: [L.sharq_kv_buffer_bytes(ctypes.byref(c), i) for i in range(-1, 5)]  # noqa: E731
    n = 8 * 16 * 2 * 128
    assert size(f8(k=None, v=None)) == [0, n, n, 16, 16, 0]
    assert size(f8(page_size=64)) == [0, 4 * n, 4 * n, 64, 64, 0]


def test_refusals(L):  # noqa: F811
    for bad, status in [(dict(k_scale=None), EINVAL), (dict(v_scale=None), EINVAL), (dict(fmt=3), EINVAL),
                        (dict(k=FAKE + 8), EALIGN), (dict(scale_rule=2), EINVAL)]:
        for call in (append, read, attention):
            assert call(L, c=f8(**bad)) == status, bad
    for b in (batch(seqs=0), batch(rows=0)):
        for c in (f8(), f8(k_scale=FAKE + 1, v_scale=FAKE + 3)):
            assert append(L, c=c, b=b) == read(L, c=c, b=b) == attention(L, c=c, b=b) == OK
    assert append(L, c=f8(k=None), b=batch(rows=0)) == EINVAL


def test_binding():
    from paper_2606_26587_amd import sharq as S
    c = S.alloc_kv_cache(4, 32, 2, 128, "fp8", "cpu", "ceil")
    assert (c.pages, c.kv_heads, c.page_size, c.head_dim, c.width) == (4, 2, 32, 128, 256)
    assert c.k.dtype == torch.float8_e4m3fn and c.k_scale.shape == (4, 2, 2) and c.k_scale.dtype == torch.uint8

    def refused(*a):
        with pytest.raises(S.SharqError) as e:
            S.KVCache("fp8", *a)
        assert e.value.status == EINVAL

    refused(c.k, c.v)
    refused(c.k, c.v, c.k_scale, None)
    refused(c.k, c.v, c.k_scale, c.v_scale[..., :1])
    refused(c.k.view(torch.uint8), c.v.view(torch.uint8), c.k_scale, c.v_scale)
    refused(c.k, c.v[:2], c.k_scale, c.v_scale)
    refused(c.k, c.v, c.k_scale, c.v_scale.to(torch.int8))


def test_plans_cover_every_tile(kv):  # noqa: F811
    """As for the other formats: a plan's workgroups take all tiles that any row sees."""
    kv.plan.restype = ctypes.c_int64
    kv.plan.argtypes = [ctypes.c_int64] * 4 + [ctypes.c_int] * 4 + [ctypes.c_int64] * 3 + [ctypes.POINTER(ctypes.c_int64)]
    rows_of, T = kv.tile_rows(), kv.tile_tokens()
    rng = np.random.default_rng(12)
    start, rg, out = (ctypes.c_int * 1)(), (ctypes.c_int * 2)(), (ctypes.c_int64 * 9)()
    big, kinds = 2 ** 31 - 1, set()
    for _ in range(800):
        seqs, most = int(rng.integers(1, 40)), int(rng.choice([1, 2, 4, 9, 40, 300, 2000]))
        n = rng.integers(0, most + 1, seqs)
        n[int(rng.integers(seqs))] = most
        lens = n + rng.integers(0, int(rng.choice([2, 100, 5000])), seqs)
        max_len = int(lens.max()) + int(rng.choice([0, 0, 17, 3000]))
        heads, group = [(8, 4), (4, 7), (1, 1), (2, 16), (1, 128), (4, 8), (3, 3)][int(rng.integers(7))]
        D = int(rng.choice([64, 128]))
        window, sinks = int(rng.choice([big, big, 1, 16, 100, 1000])), int(rng.choice([0, 1, 4, 64, 300, big]))
        prefix = int(rng.choice([0, 0, 16, 256, 1024]))
        prefix = prefix if prefix <= max_len else 0
        kv.plan(seqs, int(n.sum()), most, max_len, heads, group, D, 2, window, sinks, prefix, out)
        few, shared, own_tiles, own_chunks, own_each, pre_tiles, pre_chunks, pre_each, slots = out
        kinds.add((few, shared))
        t0, used = prefix if shared else 0, 0
        for i in range(seqs):
            base, length = int(lens[i] - n[i]), int(lens[i])
            if few:
                assert n[i] * group <= 16 * few
                if n[i]:
                    assert kv.span(t0, length, base, length - 1, window, sinks, 64, start, rg, 0) <= own_chunks * own_each
                continue
            for r0 in range(0, int(n[i]) * group, rows_of):
                last = min(int(n[i]) * group, r0 + rows_of) - 1
                used += 1
                assert kv.span(t0, length, base + r0 // group, base + last // group, window, sinks, T, start, rg,
                               0) <= own_chunks * own_each
        assert few or used <= own_tiles
        assert not shared or -(-prefix // T) <= pre_chunks * pre_each
    assert {0, 1} <= {k[0] for k in kinds}


def test_append_work_split(tmp_path):
    """Every block that a call writes is found by exactly one unit of rows, whatever the sequences."""
    (tmp_path / "s.cpp").write_text('#include "sharq_kv.hpp"\nextern "C" {\n'
                                    "int group(int64_t m) { return sharq::kv_append8_group(m); }\n"
                                    "int64_t blocks(int64_t r, int64_t m, int q, int h, int D) { return "
                                    "sharq::kv_append8_blocks(r, m, q, h, D); }\n"
                                    "int64_t queries(int64_t r, int q, int D) { return sharq::kv_append8_queries(r, q, D); }\n"
                                    "int parts(int h) { return sharq::kv_append8_parts(h); }\n}\n")
    so = str(tmp_path / "s.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2606_26587_amd", "csrc"),
                    str(tmp_path / "s.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.blocks.restype = lib.queries.restype = ctypes.c_int64
    lib.blocks.argtypes = [ctypes.c_int64, ctypes.c_int64] + [ctypes.c_int] * 3
    lib.queries.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.c_int]
    lib.group.argtypes = [ctypes.c_int64]
    rng = np.random.default_rng(3)
    for _ in range(300):
        seqs, most = int(rng.integers(1, 9)), int(rng.choice([1, 3, 16, 31, 32, 33, 100]))
        n = rng.integers(0, most + 1, seqs)
        lens = np.maximum(n + rng.integers(-3, 40, seqs), 0)
        offs = np.concatenate([[0], np.cumsum(n)])
        rows, g = int(offs[-1]) + int(rng.integers(0, 4)), lib.group(most)
        heads, q = int(rng.integers(1, 9)), int(rng.integers(0, 9))
        assert lib.parts(heads) * 4 >= 2 * heads and lib.queries(rows, q, 64) * 256 >= rows * -(-q // 2) * 4
        units = (lib.blocks(rows, most, q, heads, 64) - lib.queries(rows, q, 64)) // lib.parts(heads)
        found = []
        for u in range(units):                       # the walk of the kernel
            row, end = u * g, min(u * g + g, rows)
            while row < end:
                s = int(np.searchsorted(offs[1:], row, side="right"))
                if s >= seqs:
                    break
                base, last = int(lens[s] - n[s]), int(offs[s + 1])
                if base + row - offs[s] < 0:
                    row = int(offs[s]) - base if -base < n[s] else last
                while row < last and row < end:
                    p = base + row - int(offs[s])
                    take = min(16 - p % 16, last - row)
                    if row == offs[s] or p % 16 == 0:
                        found.append((s, p // 16, p, take))
                    row += take
        want = set()
        for s in range(seqs):
            for p in range(max(int(lens[s] - n[s]), 0), int(lens[s])):
                want.add((s, p // 16))
        assert len(found) == len(want) and {f[:2] for f in found} == want
        assert sum(f[3] for f in found) == sum(min(int(a), int(b)) for a, b in zip(n, lens))
