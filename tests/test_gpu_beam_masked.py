"""Beam search's choice where most logits are equal or masked: results, and that such rows are not read over and over."""

import numpy as np
import pytest
import torch

from paper_2606_26587_amd import sharq as S
from test_gpu_beam import TYPES, check
from test_gpu_kv import DEV

pytestmark = pytest.mark.gpu


def normal(groups, beams, vocab, dtype, seed):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((groups, beams, vocab)) * 2.5).to(TYPES[dtype]).to(DEV)
    return x, -1 - rng.random((groups, beams)).cumsum(1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("beams,vocab,left", [(1, 30000, 3), (4, 128256, 10), (8, 9001, 1), (17, 40000, 40), (32, 152064, 10),
                                              (32, 20000, 1000)])
def test_few_tokens_left_by_a_mask_of_the_lowest_value(beams, vocab, left, dtype):
    x, scores = normal(1, beams, vocab, dtype, vocab + left)
    gone = np.ones(vocab, bool)
    gone[np.random.default_rng(left).permutation(vocab)[:left]] = False
    x[..., torch.from_numpy(gone).to(DEV)] = torch.finfo(x.dtype).min
    check(x, scores)


@pytest.mark.parametrize("seed", range(8))
def test_equal_logits_in_lanes_with_and_without_any(seed):
    """Runs of 8 columns, a lane's 16 bytes, hold one of a few values or nothing, by turns of different density: lists
    fill up with equal entries, over several turns and within one."""
    rng = np.random.default_rng(seed)
    beams, vocab = [(32, 152064), (32, 90001), (8, 152064), (20, 60007)][seed % 4]
    rows = np.full((beams, -(-vocab // 2048), 256, 8), -np.inf)
    for b in range(beams):
        for t in range(rows.shape[1]):
            lanes = rng.random(256) < rng.choice([0.1, 0.3, 0.5, 0.9]) * (rng.random() < 0.9)
            rows[b, t, lanes] = rng.choice([0.0, 0.0, 0.0, 0.5, -1.0], (int(lanes.sum()), 1))
            if seed >= 4:   # within a lane as well
                rows[b, t][rng.random((256, 8)) < 0.3] = -np.inf
    x = torch.from_numpy(rows.reshape(beams, -1)[None, :, :vocab].copy()).to(torch.bfloat16).to(DEV)
    check(x, -np.arange(float(beams))[None] * 1e-3 - 1)


@pytest.mark.parametrize("beams", [24, 32])
def test_more_logits_reach_the_bound_than_the_list_holds(beams):
    """All of a lane's 32 logits are among the row's largest, for as many lanes as there are beams; no two are equal."""
    vocab = 40000
    rng = np.random.default_rng(beams)
    x = rng.standard_normal((1, beams, vocab))
    for b in range(beams):
        for lane in rng.permutation(64)[:beams + 6]:
            for k in range(8):
                at = lane * 4 + 256 * k + 2048 * int(rng.integers(0, 8))
                x[0, b, at:at + 4] = 50 + rng.permutation(4096)[:4] / 64
    check(torch.from_numpy(x).float().to(DEV), -np.arange(float(beams))[None] - 1)


def ms(f, n=5):
    f()
    times = []
    for _ in range(7):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(n):
            f()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b) / n)
    return sorted(times)[3]


def test_masked_rows_are_read_once_like_others():
    """10 tokens of 152064 left, 32 beams: what a walk for each beam takes (28 times the unmasked call, when it was made)
    against one.  A walk reads at least two rows' worth beside the lists' few lines, so a factor of 6 tells them apart."""
    x, scores = normal(1, 32, 152064, "bf16", 1)
    x, t = x[0], torch.tensor(scores, dtype=torch.float32, device=DEV)
    free = ms(lambda: S.sharq_beam_select(x, t))
    gone = torch.ones(152064, dtype=torch.bool, device=DEV)
    gone[::15207] = False
    y = x.masked_fill(gone, torch.finfo(x.dtype).min)
    assert ms(lambda: S.sharq_beam_select(y, t)) < 6 * free
