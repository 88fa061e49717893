"""README's examples: what they call with what, and the step of beam search run as it stands."""

import ast
import os
import re

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def blocks():
    with open(os.path.join(ROOT, "README.md")) as f:
        return re.findall(r"```python\n(.*?)```", f.read(), re.S)


def beam_block():
    found = [b for b in blocks() if "sharq_beam_reorder" in b]
    assert len(found) == 1
    return found[0]


def test_blocks_are_python():
    for b in blocks():
        ast.parse(b)


def test_requests_whose_tables_are_reordered_name_the_pages_they_own():
    """Behind a reorder several rows of a page table name the same page: what goes back to the pool has to be taken from
    another table, which is not reordered."""
    calls = [n for n in ast.walk(ast.parse(beam_block())) if isinstance(n, ast.Call)]
    name = lambda c: getattr(c.func, "attr", "")  # noqa: E731
    requests = [c for c in calls if name(c) == "KVRequests"]
    reorders = [c for c in calls if name(c) == "sharq_beam_reorder"]
    assert requests and reorders
    for c in requests:
        own = {k.arg: k.value for k in c.keywords}.get("own_table")
        assert isinstance(own, ast.Name)
        for r in reorders:
            used = [a.id for a in [*r.args, *(k.value for k in r.keywords)] if isinstance(a, ast.Name)]
            assert own.id not in used


@pytest.mark.gpu
def test_a_step_as_the_readme_has_it_keeps_the_pool_whole():
    """Two groups of three beams, of which all go on from one: every page comes back once when they end."""
    from paper_2606_26587_amd import sharq as S
    dev, groups, beams, page, max_len, vocab, hkv, D = "cuda", 2, 3, 64, 256, 50, 1, 64
    seqs, cols, n = groups * beams, max_len // page, 150
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)  # noqa: E731
    pages = seqs * cols
    env = dict(S=S, pages=pages, lens=z(seqs), add=z(seqs) + n, held=z(seqs), row_offsets=z(seqs + 1),
               page_table=z(seqs, cols) - 1, own_table=z(seqs, cols) - 1, rows=seqs * n, max_len=max_len, eos=0,
               ids=z(seqs, max_len), done=torch.zeros((groups, beams), dtype=torch.uint8, device=dev),
               logits=torch.from_numpy(np.random.default_rng(0).standard_normal((seqs, vocab))).to(dev, torch.float32),
               scores=torch.tensor([[-90.0, 0.0, -90.0], [-90.0, -90.0, 0.0]], device=dev),
               caches=[S.alloc_kv_cache(pages, page, hkv, D, "bf16") for _ in "ab"])
    exec(compile(beam_block(), "README.md", "exec"), env)
    assert env["parents"].tolist() == [[1] * 3, [2] * 3] and env["lens"].tolist() == [n] * seqs
    table = env["page_table"].cpu().numpy().reshape(groups, beams, cols)
    assert (table[:, :, :2] == table[:, :1, :2]).all()             # whole pages are shared,
    assert all(len(set(t[:, 2])) == beams for t in table)          # the one that is written on is not
    env["lens"].zero_(), env["add"].zero_()
    S.sharq_kv_assign(env["pool"], env["req"])
    assert int(env["pool"].count) == pages and sorted(env["pool"].free_pages.tolist()) == list(range(pages))
