"""The scale of a block of an E4M3 cache whose first tokens were never stored: the tokens that come behind them have a
scale of their own, wherever the page's byte is no scale (cleared, or never written)."""

import numpy as np
import pytest
import torch

import kv8_ref as K
import kv_ref as R
from paper_2606_26587_amd import sharq as S
from test_gpu_kv import DEV, tables

pytestmark = pytest.mark.gpu


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def u8(t):
    return t.cpu().view(torch.uint8).numpy()


@pytest.mark.parametrize("stale", [0, 9, 248, 255])
@pytest.mark.parametrize("why", ["angle below the tables", "angle past the tables", "absent page"])
@pytest.mark.parametrize("D,page,first,new", [(64, 16, 1, 1), (128, 32, 15, 1), (128, 32, 5, 40), (64, 64, 37, 2)])
def test_tokens_behind_those_left_out(D, page, first, new, why, stale):
    hkv, angles = 2, 100
    n, start = first + new, first // 16 * 16            # the block that both calls have tokens of begins at `start`
    cols = -(-n // page)
    table = np.arange(1, cols + 1, dtype=np.int32)[None]
    codes = torch.full((cols + 1, hkv, page, D), 0x35, dtype=torch.uint8, device=DEV)
    scales = torch.full((cols + 1, hkv, page // 16), stale, dtype=torch.uint8, device=DEV)
    cache = S.KVCache("fp8", codes.view(torch.float8_e4m3fn), codes.clone().view(torch.float8_e4m3fn), scales,
                      scales.clone(), "ceil")
    x = R.bf16(np.random.default_rng(first).standard_normal((n, 2 * hkv * D))).to(DEV)
    k, v = x[:, :hkv * D], x[:, hkv * D:]
    cos, sin = (torch.from_numpy(t).to(DEV) for t in tables(angles, D))
    out = {"angle below the tables": -1, "angle past the tables": angles}.get(why)
    there = i32(*table[0])[None]
    S.sharq_kv_append(None, k[:first], v[:first], cache,
                      S.KVBatch(i32(0, first), i32(first), there if out is not None else there * 0 - 1, first, first, n),
                      cos, sin, positions=None if out is None else torch.full((first,), out, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for t, was in ((cache.k, 0x35), (cache.v, 0x35), (cache.k_scale, stale), (cache.v_scale, stale)):
        assert (u8(t) == was).all()
    S.sharq_kv_append(None, k[first:], v[first:], cache, S.KVBatch(i32(0, new), i32(n), there, new, new, n), cos, sin)
    torch.cuda.synchronize()

    xs = x.float().cpu().numpy().reshape(n, 2 * hkv, D)
    pos = np.arange(n)
    y = R.rotate32(xs[:, :hkv], cos.cpu().numpy()[pos], sin.cpu().numpy()[pos])
    want = [np.full((cols + 1, hkv, page, D), 0x35, np.uint8) for _ in "kv"] + \
           [np.full((cols + 1, hkv, page // 16), stale, np.uint8) for _ in "kv"]
    # without tokens before them, as the definition has it: the call's rows as those of blocks that begin with them
    for b in range(start // 16, -(-n // 16)):
        p = pos[max(first, 16 * b):16 * b + 16]
        pg, at = table[0, 16 * b // page], 16 * b % page // 16
        for x_, c, s in ((y, want[0], want[2]), (xs[:, hkv:], want[1], want[3])):
            for h in range(hkv):
                rows = x_[p, h].astype(np.float64)
                e = K.exponent(np.abs(rows).max(), "ceil")
                c[pg, h, p % page] = K.encode(rows * 2.0 ** -e)
                s[pg, h, at] = e + 127
    for got, exp, name in zip((cache.k, cache.v, cache.k_scale, cache.v_scale), want, ("k", "v", "k_scale", "v_scale")):
        assert np.array_equal(u8(got), exp), name


def test_a_scale_that_is_there_stays(D=64, page=16):
    """The largest and the least scale that an append can leave count like any other."""
    for byte, rows in ((247, 1), (10, 1)):
        codes = torch.full((1, 1, page, D), 0x38, dtype=torch.uint8, device=DEV)   # ones
        scales = torch.full((1, 1, 1), byte, dtype=torch.uint8, device=DEV)
        cache = S.KVCache("fp8", codes.view(torch.float8_e4m3fn), codes.clone().view(torch.float8_e4m3fn), scales,
                          scales.clone(), "ceil")
        x = torch.full((1, D), 2.0 ** -112 if byte == 10 else 2.0 ** 120, dtype=torch.bfloat16, device=DEV)
        S.sharq_kv_append(None, x, x, cache, S.KVBatch(i32(0, 1), i32(6), i32(0)[None], 1, 1, 6))
        k, v = S.sharq_kv_read(cache, S.KVBatch(i32(0, 6), i32(6), i32(0)[None], 6, 6, 6))
        torch.cuda.synchronize()
        want = torch.full((6, D), 2.0 ** (byte - 127), dtype=torch.float64)
        want[5] = 2.0 ** -112 if byte == 10 else 2.0 ** 120
        assert torch.equal(k.double().cpu(), want) and torch.equal(v.double().cpu(), want)
        assert (u8(cache.k_scale) == byte).all()
