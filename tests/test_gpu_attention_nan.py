"""A NaN that a row sees makes that row NaN, whether or not the call splits its
tokens over workgroups, and no row of another sequence or key/value head.  (The
results of such inputs are not specified; that they do not pass for numbers is.)"""

import numpy as np
import pytest
import torch

import kv_ref as R
from paper_2606_26587_amd import sharq as S
from test_gpu_attention import setup

pytestmark = pytest.mark.gpu

HQ, HKV, D, PAGE = 8, 2, 128, 16
G = HQ // HKV


def spoil(pool, scale, page, head, slot, at):
    """NaN into one value of a bf16 row, or into the block of 32 that holds it."""
    if scale is None:
        pool[page, head, slot, at] = float("nan")
        return slice(at, at + 1)
    scale[page, head, slot, at // 32] = 0xFF
    return slice(at // 32 * 32, at // 32 * 32 + 32)


CASES = [
    # rows, lengths, prefix, token with the NaN (of sequence 0), whether the call splits
    ([1, 1], [9000, 50], 0, 4321, True),
    ([2, 1], [3000, 900], 0, 0, True),
    ([30, 3], [3000, 70], 0, 2960, True),
    ([1, 1], [40, 20], 0, 39, False),
    ([200, 9], [200, 9], 0, 100, False),
    ([1, 1, 1], [3000, 2200, 2100], 2048, 2500, True),
    ([1, 1, 1], [3000, 2200, 2100], 2048, 700, True),       # in the prefix: every sequence's
    ([20, 3], [1500, 1100], 1024, 1300, True),
]


@pytest.mark.parametrize("fmt", ["bf16", "mx"])
@pytest.mark.parametrize("what", ["key", "value", "query"])
@pytest.mark.parametrize("per,lens,prefix,t,split", CASES)
def test_a_nan_shows(per, lens, prefix, t, split, what, fmt):
    batch, offsets, ln, table, cache, q = setup(per, lens, PAGE, HQ, HKV, D, fmt)
    pt = batch.page_table[0, :prefix // PAGE].contiguous() if prefix else None
    size = S.attention_workspace_bytes(cache, batch, HQ, prefix_len=prefix)
    assert (size > 0) == split

    def call():
        lse = torch.full((batch.rows, HQ), 9.0, device=q.device)
        out = S.sharq_attention(q, cache, batch, prefix_table=pt, prefix_len=prefix, lse=lse)
        torch.cuda.synchronize()
        return out.float().cpu().reshape(batch.rows, HQ, D), lse.cpu()

    clean, clean_lse = call()
    assert torch.isfinite(clean).all() and torch.isfinite(clean_lse).all()
    head, dim = 1, 70
    seq, pos = R.positions(offsets, ln, batch.rows)
    sees = torch.from_numpy((pos >= t) & ((seq == 0) | (t < prefix)))
    heads = slice(head * G, head * G + G)
    hit = slice(0, D)
    if what == "query":
        row = int(np.flatnonzero(seq == 0)[-1])
        q[row, (head * G + 2) * D + dim] = float("nan")
        sees, heads = torch.arange(batch.rows) == row, slice(head * G + 2, head * G + 3)
    else:
        pool, scale = (cache.k, cache.k_scale) if what == "key" else (cache.v, cache.v_scale)
        block = spoil(pool, scale, int(table[0, t // PAGE]), head, t % PAGE, dim)
        if what == "value":
            hit = block
    got, lse = call()
    assert sees.any()
    assert torch.isnan(got[sees][:, heads, hit]).all()
    if what == "value":                                     # the other columns, and the weights, have no part in it
        rest = torch.ones(D, dtype=torch.bool)
        rest[hit] = False
        assert torch.equal(got[sees][:, heads][..., rest], clean[sees][:, heads][..., rest])
        assert torch.equal(lse, clean_lse)
    else:
        assert torch.isnan(lse[sees][:, heads]).all()
    # other key/value heads, and the other sequences where the NaN is none of theirs
    other = torch.ones(HQ, dtype=torch.bool)
    other[head * G:head * G + G] = False
    assert torch.equal(got[:, other], clean[:, other]) and torch.equal(lse[:, other], clean_lse[:, other])
    if what != "query" and t >= prefix:
        apart = torch.from_numpy(seq != 0)
        assert torch.equal(got[apart], clean[apart]) and torch.equal(lse[apart], clean_lse[apart])
