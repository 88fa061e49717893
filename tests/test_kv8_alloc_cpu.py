"""A new E4M3 cache holds no scale, whatever its memory held before."""

import torch

from paper_2606_26587_amd import sharq as S


def test_scales_of_a_new_cache_are_cleared(monkeypatch):
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: empty(*a, **kw).view(torch.uint8).fill_(0xF0).view(kw["dtype"]))
    c = S.alloc_kv_cache(3, 32, 2, 64, "fp8", "cpu")
    assert not c.k_scale.any() and not c.v_scale.any() and c.k_scale.shape == c.v_scale.shape == (3, 2, 2)
    assert S.alloc_kv_cache(3, 32, 2, 64, "bf16", "cpu").k_scale is None
