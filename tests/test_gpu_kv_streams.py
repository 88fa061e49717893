"""Calls on a stream of their own without buffers given: what they allocate lies
in that stream's blocks, and they compute what a call on the current stream does."""

import numpy as np
import pytest
import torch

import kv_ref as R
from paper_2606_26587_amd import sharq as S
from test_gpu_attention import setup
from test_gpu_kv import DEV

pytestmark = pytest.mark.gpu


def stream_of(t):
    """Handle of the stream whose block of the allocator holds the tensor."""
    at = t.data_ptr()
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= at < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("no block holds the tensor")


@pytest.mark.parametrize("fmt", ["bf16", "mx"])
def test_cache_and_attention_outputs(fmt):
    per, lens, hq, hkv, D = [1, 3], [3000, 40], 8, 2, 128
    batch, offsets, ln, table, cache, q = setup(per, lens, 16, hq, hkv, D, fmt)
    kv = R.bf16(np.random.default_rng(0).standard_normal((batch.rows, hkv * D))).to(DEV)
    side = torch.cuda.Stream()

    def step(stream):
        turned = S.sharq_kv_append(q, kv, kv, cache, batch, stream=stream)
        return (turned, S.sharq_attention(turned, cache, batch, stream=stream),
                *S.sharq_kv_read(cache, batch, stream=stream))

    want = step(None)
    torch.cuda.synchronize()
    for _ in range(2):
        for t in [torch.empty_like(w) for w in want]:   # blocks of the current stream to take by mistake
            del t
        got = step(side)
        side.synchronize()
        for g, w in zip(got, want):
            assert torch.equal(g, w) and stream_of(g) == side.cuda_stream
            assert stream_of(w) == torch.cuda.current_stream().cuda_stream
        del got


def test_linear_outputs():
    """The layer's linears, whose buffers are their stream's as well."""
    x = R.bf16(np.random.default_rng(0).standard_normal((5, 256))).to(DEV)
    side = torch.cuda.Stream()

    def step(stream):
        w = S.sharq_quantize_weight(x[:, :256].repeat(26, 1)[:128].contiguous(), stream=stream)
        act, y = S.sharq_prepare_linear(x, None, w, stream=stream)
        p, h = S.sharq_prepare_residual(x, x, None, stream=stream)
        return w.codes, act.dn_codes, y, p.dn_codes, h, S.sharq_linear(p, w, stream=stream)

    want = step(None)
    torch.cuda.synchronize()
    got = step(side)
    side.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w) and stream_of(g) == side.cuda_stream
