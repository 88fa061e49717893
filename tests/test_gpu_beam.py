"""Beam search's choice, the reordering behind it and the copies of pages on the GPU."""

import numpy as np
import pytest
import torch

import kv8_ref as K
import kv_ref as KR
import serve_ref as R
from paper_2606_26587_amd import sharq as S
from test_gpu_kv import DEV, empty_cache
from test_gpu_kv import tables as KR_tables

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}

# How far a score may be from the definition in 64 bits, besides its own rounding to fp32.  A term e^(x - ref) of the sum
# has x - ref rounded (2^-24 of it, at most 8 above the reference: for terms above the reference 2^-21), its product with
# log2 e (2^-24 of at most 11.6, and as much for the constant: 2^-20 together) and the exponential (2^-23); six sums in
# fp32 (2^-24 each); all later ones in 64 bits.  Terms below the reference by d have errors of 2^-22 d + 2^-22, weighted by
# e^-d: less.  Together below 2^-19 of the sum, and so of its logarithm.
LSE = 2.0 ** -19


def run(x, scores, done=None, eos=-1, **kw):
    """x [groups, beams, vocab] tensor on the device (last two may be strided), scores [groups, beams] numpy."""
    groups, beams, vocab = x.shape
    t = lambda a, d: None if a is None else torch.tensor(np.asarray(a), dtype=d, device=DEV)  # noqa: E731
    logits = x.reshape(groups * beams, vocab) if x.is_contiguous() else x.flatten(0, 1)
    return S.sharq_beam_select(logits, t(scores, torch.float32), done=t(done, torch.uint8), eos=eos, **kw)


def check(x, scores, done=None, eos=-1, out=None):
    groups, beams, vocab = x.shape
    got = run(x, scores, done, eos) if out is None else out
    torch.cuda.synchronize()
    gs, gp, gt, gd = (None if t is None else t.cpu().numpy() for t in got)
    xd = x.double().cpu().numpy()
    scores = np.asarray(scores, np.float32)
    for g in range(groups):
        dn = None if done is None else np.asarray(done)[g]
        want = R.candidates(xd[g], scores[g], dn, eos, beams)
        of = {(b, v): c for c, b, v in want}
        n = min(beams, len(want))
        chosen = [(int(gp[g, r]), int(gt[g, r])) for r in range(n)]
        assert len(set(chosen)) == n
        for r in range(n):
            assert chosen[r] in of, (g, r, chosen[r])
            c = of[chosen[r]]
            # the r-th best, up to the errors of two sums
            assert abs(c - want[r][0]) <= 2 * LSE or c == want[r][0], (g, r, c, want[r])
            assert abs(float(gs[g, r]) - c) <= LSE + abs(c) * 2.0 ** -24 or float(gs[g, r]) == np.float32(c), (g, r)
        for b in range(beams):   # within a beam the order is exact
            mine = [v for p, v in chosen if p == b]
            best = [v for _, p, v in want if p == b][:len(mine)]
            assert mine == best, (g, b, mine, best)
        for r in range(n, beams):
            assert np.isneginf(gs[g, r]) and gt[g, r] == -1 and gp[g, r] == r
        if dn is not None:
            for r in range(beams):
                assert gd[g, r] == int(bool(dn[gp[g, r]]) or gt[g, r] == eos)
    return gs, gp, gt, gd


def logits(groups, beams, vocab, dtype, seed=0, scale=2.5):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((groups, beams, vocab)) * scale
    x[..., rng.integers(0, vocab, max(1, vocab // 5000))] += 8
    return torch.from_numpy(x).to(TYPES[dtype]).to(DEV), -20 - rng.random((groups, beams)).cumsum(1)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("groups,beams,vocab", [
    (1, 1, 1), (2, 1, 9), (1, 4, 5), (3, 8, 3), (2, 5, 64), (1, 4, 2047), (1, 4, 2049), (2, 3, 8191), (1, 2, 8193),
    (1, 16, 152064), (1, 20, 152064), (1, 24, 152064), (1, 32, 152064), (1, 3, 700000),   # many parts of a row
    (3, 8, 50257), (1, 32, 9000), (2, 24, 20001), (5, 2, 128256), (1, 4, 152064), (1, 16, 33333), (130, 8, 1000)])
def test_choice(groups, beams, vocab, dtype):
    x, scores = logits(groups, beams, vocab, dtype, seed=vocab + beams)
    check(x, scores)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_rows_with_a_stride_and_at_any_element(pad, dtype):
    x, scores = logits(3, 4, 5001, dtype, seed=pad)
    wide = torch.full((12, 5001 + pad), float("nan"), dtype=x.dtype, device=DEV)
    wide[:, :5001] = x.flatten(0, 1)
    flat = torch.full((12 * (5001 + pad) + 5,), float("nan"), dtype=x.dtype, device=DEV)
    odd = flat[5:].view(12, 5001 + pad)
    odd.copy_(wide)
    t = torch.tensor(scores, dtype=torch.float32, device=DEV)
    want = check(x, scores)
    for y in (wide, odd):
        got = S.sharq_beam_select(y[:, :5001], t)
        for a, b in zip(got[:3], want[:3]):
            assert np.array_equal(a.cpu().numpy(), b)


@pytest.mark.parametrize("beams", [1, 3, 8])
def test_beams_that_are_done(beams):
    rng = np.random.default_rng(beams)
    x, scores = logits(6, beams, 3000, "bf16", seed=beams)
    done = rng.random((6, beams)) < 0.5
    done[0], done[1] = True, False
    scores[2] += 18                        # ended beams far ahead of the others
    scores[3][done[3]] -= 100              # and far behind
    x[4, :, 77] = 30                       # beams that end now
    check(x, scores, done.astype(np.uint8), eos=77)
    check(x, scores, (done * 255).astype(np.uint8), eos=2999)
    check(x, scores, np.zeros((6, beams), np.uint8), eos=0)


def test_ties_go_to_the_lowest_index():
    """Equal rows and equal scores: beams are the same to the last bit, and the order is by beam and token."""
    for dtype, vocab in (("bf16", 5001), ("fp32", 5001), ("fp16", 8), ("bf16", 20000)):
        x, _ = logits(2, 1, vocab, dtype, seed=vocab)
        x = x.expand(2, 6, vocab).contiguous()
        gs, gp, gt, _ = check(x, np.full((2, 6), -3.25))
        for g in range(2):
            best = int(torch.argmax(x[g, 0].float()))
            assert list(gp[g]) == list(range(6)) and (gt[g] == best).all() and len(set(gs[g])) == 1


@pytest.mark.parametrize("vocab", [5, 64, 2048, 9001, 30000])
@pytest.mark.parametrize("kind", ["same", "rising", "falling", "two", "blocks"])
def test_rows_full_of_ties_and_sorted_rows(kind, vocab):
    v = np.arange(vocab)
    row = {"same": np.zeros(vocab), "rising": v / vocab * 3.0, "falling": -v / vocab * 3.0, "two": (v % 2) * 1.0,
           "blocks": v // 300 % 7 * 0.5}[kind]
    x = torch.from_numpy(np.broadcast_to(row, (1, 8, vocab)).copy()).to(torch.bfloat16).to(DEV)
    check(x, -np.arange(8.0)[None] * 1e-3 - 1)
    check(x.float(), np.array([[-np.inf] * 7 + [0.0]]))


def test_masked_tokens_and_rows_without_any():
    inf = float("inf")
    x, scores = logits(7, 4, 4000, "fp32", seed=9)
    x[0, :, 10:] = -inf                                # ten tokens left
    x[1, 1] = -inf                                     # a beam with none
    x[2] = -inf                                        # a group with none
    x[3, :, 1:] = -inf                                 # as many candidates as beams
    x[4, :2] = -inf
    x[4, 2:, 1:] = -inf                                # fewer candidates than beams
    x[5, :, 5:] = torch.finfo(torch.float32).min       # a mask of the type's lowest value
    x[6, 2] = torch.finfo(torch.float32).min           # a row of nothing else
    check(x, scores)
    y, scores = logits(2, 4, 4000, "bf16", seed=10)
    y[0, :, 100:] = torch.finfo(torch.bfloat16).min
    y[1] = torch.finfo(torch.bfloat16).min
    check(y, scores)


def test_the_first_step_and_beams_without_a_score():
    x, scores = logits(3, 5, 2000, "bf16", seed=3)
    scores[:, 1:] = -np.inf
    check(x, scores)
    scores[1, 0], scores[2, 0], scores[2, 3] = -np.inf, np.nan, -4
    check(x, scores)
    scores[0, 2], scores[1, 1], scores[2, 1] = np.inf, -1, np.inf
    check(x, scores)
    check(x, scores, np.array([[0, 0, 1, 0, 0], [1, 1, 0, 0, 0], [1, 1, 0, 1, 0]], np.uint8), eos=3)
    # sums that lose the logits: within a beam these decide
    for huge in (-1e9, -1e30, 3e38):
        check(x.float(), np.full((3, 5), huge))
        check(x.float() * 1e-3, np.array([[huge, -np.inf, -np.inf, -np.inf, -np.inf]] * 3))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("nan")])
@pytest.mark.parametrize("at", [0, 7, 2500, 29999])
def test_a_beam_with_a_nan_or_infinity_has_no_candidate(bad, at):
    x, scores = logits(2, 3, 30000, "fp32", seed=1)
    x[0, 1, at] = bad
    x[1, 2] = bad
    gs, gp, _, _ = check(x, scores)
    assert not (gp[0] == 1).any() and not (gp[1] == 2).any() and np.isfinite(gs).all()


def test_large_and_small_logits():
    x, scores = logits(3, 4, 10000, "fp32", seed=2, scale=1e4)
    check(x, scores)
    x, scores = logits(2, 4, 10000, "fp32", seed=2, scale=1e-6)
    check(x, scores)
    x, scores = logits(1, 4, 20000, "fp16", seed=2, scale=6000)
    check(x.clamp(-65000, 65000), scores)
    x, scores = logits(1, 2, 3000, "fp32", seed=5)
    x[0, 0, 5], x[0, 0, 2999], x[0, 1, 0] = -3.4e38, 3.3e38, 3.4e38
    check(x, scores)


def test_rising_references():
    """Every turn's largest logit passes the one before by more than the step, up and down."""
    for sign in (1, -1):
        row = sign * (np.arange(60000) // 2048) * 9.5 + np.random.default_rng(0).standard_normal(60000)
        x = torch.from_numpy(np.stack([row, row[::-1].copy()])[None]).float().to(DEV)
        check(x, [[-1.0, -2.0]])


def test_in_place_on_a_stream_with_a_workspace_and_captured():
    groups, beams, vocab, eos = 4, 6, 12000, 500
    ws = torch.empty(S.beam_workspace_bytes(groups, beams, vocab), dtype=torch.uint8, device=DEV)
    scores = torch.zeros((groups, beams), device=DEV)
    done = torch.zeros((groups, beams), dtype=torch.uint8, device=DEV)
    x = torch.zeros((groups * beams, vocab), dtype=torch.bfloat16, device=DEV)
    parents, tokens = (torch.zeros((groups, beams), dtype=torch.int32, device=DEV) for _ in "pt")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        S.sharq_beam_select(x, scores, done, eos, scores, parents, tokens, done, ws)
    for step in range(4):
        y, s = logits(groups, beams, vocab, "bf16", seed=step)
        d = np.random.default_rng(step).random((groups, beams)) < 0.3
        x.copy_(y.flatten(0, 1))
        scores.copy_(torch.from_numpy(s))
        done.copy_(torch.from_numpy(d))
        torch.cuda.synchronize()
        graph.replay()
        check(y, s, d.astype(np.uint8), eos, out=(scores, parents, tokens, done))
        eager = run(y, s, d.astype(np.uint8), eos, stream=side)
        side.synchronize()
        for a, b in zip(eager, (scores, parents, tokens, done)):
            assert torch.equal(a, b)


# ---------------------------------------------------------------------------
# Reordering
# ---------------------------------------------------------------------------

def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def reorder_case(groups, beams, page, lens, cols, id_cols, seed, parents=None, in_place=False, pad=2):
    rng = np.random.default_rng(seed)
    table = rng.permutation(groups * beams * (cols + 1))[:groups * beams * cols].reshape(groups, beams, cols)
    ids = rng.integers(0, 10 ** 6, (groups, beams, id_cols))
    tokens = rng.integers(0, 10 ** 6, (groups, beams))
    if parents is None:
        parents = np.minimum(rng.integers(0, beams, (groups, beams)), rng.integers(0, beams, (groups, beams)))

    def wide(x, fill):
        t = torch.full((groups * beams, x.shape[2] + pad), fill, dtype=torch.int32, device=DEV)
        t[:, :x.shape[2]] = i32(x.reshape(groups * beams, -1))
        return t

    t_table, t_ids = wide(table, -5), wide(ids, -6)
    to = t_table if in_place else torch.full_like(t_table, -5)
    ido = t_ids if in_place else torch.full_like(t_ids, -6)
    per = np.repeat(lens, beams)
    per.reshape(groups, beams)[:, 1:] = 10 ** 8           # the first of a group counts
    copies = S.sharq_beam_reorder(i32(parents), i32(per), t_table[:, :cols], page, tokens=i32(tokens),
                                  ids=t_ids[:, :id_cols], table_out=None if in_place else to[:, :cols],
                                  ids_out=None if in_place else ido[:, :id_cols])
    torch.cuda.synchronize()
    to, ido, copies = (t.cpu().numpy().reshape(groups, beams, -1) for t in (to, ido, copies))
    assert (to[..., cols:] == -5).all() and (ido[..., id_cols:] == -6).all()
    for g in range(groups):
        n = int(lens[g])
        new, want, out = R.reorder(parents[g], n, page, table[g], ids[g], tokens[g])
        assert np.array_equal(to[g, :, :cols], new), g
        assert [tuple(c) for c in copies[g]] == [tuple(c) for c in want], g
        out = np.array(out)
        if not in_place:
            out[:, min(n + 1, id_cols):] = -6
        assert np.array_equal(ido[g, :, :id_cols], out), g
        if n % page and n // page < cols:                 # nobody shares a page that is written on
            assert len(set(to[g, :, n // page])) == beams


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("groups,beams,page,cols", [(1, 1, 16, 3), (3, 4, 16, 9), (2, 8, 32, 70), (5, 32, 16, 130),
                                                    (40, 3, 64, 65), (2, 2, 1024, 2)])
def test_reorder(groups, beams, page, cols, in_place):
    rng = np.random.default_rng(cols)
    top = cols * page
    for i, lens in enumerate([rng.integers(0, top + 1, groups), np.full(groups, top), np.full(groups, 0),
                              np.full(groups, page), np.full(groups, top - 1), np.full(groups, top // 2 + 1)]):
        reorder_case(groups, beams, page, lens, cols, min(top + 3, 900), i, in_place=in_place)


def test_reorder_of_given_parents():
    for parents in ([[0, 0, 0, 0]], [[3, 3, 3, 3]], [[1, 0, 3, 2]], [[0, 1, 2, 3]], [[2, 2, 1, 1]], [[3, 0, 0, 3]]):
        reorder_case(1, 4, 16, [37], 4, 50, 1, np.array(parents), in_place=True)
        reorder_case(1, 4, 16, [48], 4, 50, 1, np.array(parents))
    reorder_case(1, 4, 16, [37], 4, 50, 1, np.array([[-9, 2 ** 31 - 1, 4, -2 ** 31]]))


def test_reorder_of_tables_or_tokens_alone_and_lengths_out_of_range():
    parents = i32([[1, 1, 0]])
    table = i32([[1, 2], [3, 4], [5, 6]])
    copies = S.sharq_beam_reorder(parents, i32([20, 20, 20]), table, 16)
    assert table.tolist() == [[3, 4], [3, 6], [1, 2]] and copies.tolist() == [[-1] * 3, [4, 6, 4], [-1] * 3]
    ids = i32([[1, 2, 3], [4, 5, 6], [7, 8, 9]])
    assert S.sharq_beam_reorder(parents, i32([2, 0, 0]), None, 16, tokens=i32([[10, 11, 12]]), ids=ids) is None
    assert ids.tolist() == [[4, 5, 10], [4, 5, 11], [1, 2, 12]]
    for n, whole in ((-3, 0), (2 ** 31 - 1, 2), (33, 2)):
        table = i32([[1, 2], [3, 4], [5, 6]])
        ids = i32([[1, 2, 3], [4, 5, 6], [7, 8, 9]])
        copies = S.sharq_beam_reorder(parents, i32([n] * 3), table, 16, tokens=i32([[10, 11, 12]]), ids=ids)
        assert (copies == -1).all() and table.tolist() == ([[3, 4], [3, 4], [1, 2]] if whole else [[1, 2], [3, 4], [5, 6]])
        assert ids.tolist() == ([[4, 5, 6], [4, 5, 6], [1, 2, 3]] if whole else [[10, 2, 3], [11, 5, 6], [12, 8, 9]])


# ---------------------------------------------------------------------------
# Copies
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["bf16", "mx", "fp8"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,hkv", [(16, 1), (16, 8), (64, 3), (128, 8), (1024, 2)])
def test_copies(page, hkv, D, fmt):
    rng = np.random.default_rng(page + hkv)
    pages = 14
    cache = empty_cache(pages, page, hkv, D, fmt)
    buffers = [t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]
    for t in buffers:
        t.view(torch.uint8).copy_(torch.from_numpy(rng.integers(0, 120, t.view(torch.uint8).shape, dtype=np.uint8)).to(DEV))
    before = [t.cpu().view(torch.uint8).numpy().copy() for t in buffers]
    copies = [(0, 1, 1), (0, 2, page), (3, 4, page - 1), (5, 5, 4), (-1, -1, -1), (6, 7, 0), (6, 8, page + 50), (3, 9, 17),
              (pages, 10, 3), (3, 2 ** 31 - 1, 3), (-2 ** 31, 11, 3), (3, 12, -8), (13, 10, page // 2 + 1)]
    S.sharq_kv_copy(cache, i32(copies))
    torch.cuda.synchronize()
    for t, want in zip(buffers, before):
        source = want.copy()
        per = page // want.shape[2]                       # tokens of an entry: a block's scale in an fp8 cache
        for s, d, n in copies:
            if 0 <= s < pages and 0 <= d < pages and s != d and n > 0:
                m = -(-min(n, page) // per)
                want[d, :, :m] = source[s, :, :m]
        assert np.array_equal(t.cpu().view(torch.uint8).numpy(), want)


def test_copies_past_32_bits():
    page, hkv, D = 1024, 8, 128
    pages = 2 ** 32 // (page * hkv * D) + 3
    cache = S.alloc_kv_cache(pages, page, hkv, D, "fp8", DEV)
    g = torch.Generator(device=DEV).manual_seed(0)
    for p in (0, pages - 1):
        for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
            u = t.view(torch.uint8)[p]
            u.copy_(torch.randint(0, 100, u.shape, generator=g, device=DEV, dtype=torch.uint8))
    S.sharq_kv_copy(cache, i32([(pages - 1, pages - 2, page), (0, 1, 100)]))
    for t in (cache.k, cache.v, cache.k_scale, cache.v_scale):
        u = t.view(torch.uint8)
        assert torch.equal(u[pages - 1], u[pages - 2])
        n = 100 if t.dim() == 4 else 7
        assert torch.equal(u[0, :, :n], u[1, :, :n])


# ---------------------------------------------------------------------------
# All of it together
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["fp8", "bf16", "mx"])
def test_beam_search_over_a_paged_cache(fmt):
    """Prompts, then 40 steps of assign, append, attention, choice, reorder and copies.  At every step the cache holds,
    for every beam, the keys and values of its tokens; the attention is that of its tokens; the choice is the best."""
    rng = np.random.default_rng(11)
    groups, beams, page, hq, hkv, D, vocab, steps = 3, 4, 16, 8, 2, 64, 300, 40
    seqs, prompts = groups * beams, [21, 16, 5]
    max_len, eos = 70, 7
    embed_q, embed_k, embed_v = (rng.standard_normal((vocab, n * D)) for n in (hq, hkv, hkv))
    head = torch.from_numpy(rng.standard_normal((hq * D, vocab)) * 0.15).float().to(DEV)
    te = [KR.bf16(e).to(DEV) for e in (embed_q, embed_k, embed_v)]
    he = [t.double().cpu().numpy() for t in te]
    pages = groups * (2 + beams * 5) + 2
    cache = S.alloc_kv_cache(pages, page, hkv, D, fmt, DEV, "ceil")
    pool = S.alloc_kv_pool(pages)
    zeros = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    cols = -(-max_len // page)
    lens, add, held, offs = zeros(seqs), zeros(seqs), zeros(seqs), zeros(seqs + 1)
    table, own = zeros(seqs, cols) - 1, zeros(seqs, cols) - 1
    ids, positions, row_seq = zeros(seqs, max_len + 1), zeros(64), zeros(64)

    def step_call(rows):
        req = S.KVRequests(lens, add, held, offs, lens, table, rows, max_len, page, own_table=own, missing=zeros(1),
                           positions=positions[:rows], row_seq=row_seq[:rows])
        S.sharq_kv_assign(pool, req)
        assert int(req.missing) == 0
        return req

    # the prompts, by the first beam of each group; the others hold the pages of the part behind the shared ones
    prompt = [rng.integers(8, vocab, n) for n in prompts]
    add.copy_(i32([n if b == 0 else 0 for n in prompts for b in range(beams)]))
    total = sum(prompts)
    batch = step_call(total).batch(max(prompts))
    tok = torch.from_numpy(np.concatenate(prompt)).to(DEV)
    S.sharq_kv_append(None, te[1][tok], te[2][tok], cache, batch)
    o = S.sharq_attention(te[0][tok], cache, batch)
    last = (offs[1:].view(groups, beams)[:, 0] - 1).long()
    x = (o[last].float() @ head).repeat_interleave(beams, 0)
    lens.copy_(i32([n for n in prompts for _ in range(beams)]))
    held.copy_(i32([-(-n // page) if b == 0 else n // page for n in prompts for b in range(beams)]))
    add.zero_()
    step_call(0)
    scores = torch.full((groups, beams), -float("inf"), device=DEV)
    scores[:, 0] = 0
    done = torch.zeros((groups, beams), dtype=torch.uint8, device=DEV)
    for g in range(groups):
        ids[g * beams, :prompts[g]] = i32(prompt[g])
    text = [[list(prompt[g])] * beams for g in range(groups)]
    n_of = list(prompts)
    for step in range(steps):
        before = (scores.cpu().numpy().copy(), done.cpu().numpy().copy())
        check(x.view(groups, beams, vocab), before[0], before[1], eos,
              out=S.sharq_beam_select(x, scores, done, eos))
        scores, parents, tokens, done = S.sharq_beam_select(x, scores, done, eos, scores_out=scores, done_out=done)
        p, t = parents.cpu().numpy(), tokens.cpu().numpy()
        text = [[text[g][p[g, b]] + [int(t[g, b])] for b in range(beams)] for g in range(groups)]
        copies = S.sharq_beam_reorder(parents, lens, table, page, tokens=tokens, ids=ids)
        S.sharq_kv_copy(cache, copies)
        got = ids.cpu().numpy().reshape(groups, beams, -1)
        for g in range(groups):
            for b in range(beams):
                assert list(got[g, b, :n_of[g] + 1]) == text[g][b]
        # the next step: the tokens that were chosen
        add.fill_(1)
        req = step_call(seqs)
        assert row_seq[:seqs].tolist() == list(range(seqs))
        n_of = [n + 1 for n in n_of]
        assert positions[:seqs].tolist() == [n_of[g] - 1 for g in range(groups) for _ in range(beams)]
        batch = req.batch(1)
        tok = tokens.flatten().long()
        S.sharq_kv_append(None, te[1][tok], te[2][tok], cache, batch)
        o = S.sharq_attention(te[0][tok], cache, batch)
        x = o.float() @ head
        # what the cache holds of each beam
        whole = S.KVBatch(i32(np.concatenate([[0], np.cumsum([n for n in n_of for _ in range(beams)])])), lens, table,
                          sum(n_of) * beams, max(n_of), max_len)
        k, v = (y.double().cpu().numpy() for y in S.sharq_kv_read(cache, whole))
        at = 0
        for g in range(groups):
            for b in range(beams):
                for y, e in ((k, he[1]), (v, he[2])):
                    want, mine = e[text[g][b]], y[at:at + n_of[g]]
                    if fmt == "bf16":
                        assert np.array_equal(mine, want)
                    elif fmt == "mx":
                        c, s = KR.mx_quantize(want.astype(np.float32).reshape(-1, hkv, D), "ceil")
                        assert np.array_equal(mine, KR.mx_values(c, s).reshape(mine.shape))
                    else:
                        # half a step, or half of the least code under a scale of the largest magnitude; a value may be
                        # rounded again where its scale grows, which is exact above the subnormal codes
                        unit = np.abs(e).max() * 2.0 ** -8 * 2
                        assert (np.abs(mine - want) <= np.maximum(np.abs(want) * 2.0 ** -4, unit * 2.0 ** -9)).all()
                if step % 13 == 0:
                    kb, vb = (y[at:at + n_of[g]].reshape(1, -1, hkv, D).swapaxes(1, 2) for y in (k, v))
                    q = he[0][text[g][b][-1]].reshape(1, hq, D)
                    scale = float(np.float32(D ** -0.5))
                    r, _, mag, size = KR.attention(q, kb, vb, [0, 1], [n_of[g]], [[0] * (n_of[g] // n_of[g])], scale)
                    tol = KR.tolerance(r, mag, size, D, scale, n_of[g], np.abs(vb).max())
                    assert (np.abs(o[g * beams + b].double().cpu().numpy().reshape(1, hq, D) - r) <= tol).all()
                at += n_of[g]
    # all sequences end: every page comes back, once
    lens.zero_()
    add.zero_()
    step_call(0)
    assert int(pool.count) == pages and sorted(pool.free_pages.tolist()) == list(range(pages))


@pytest.mark.parametrize("fmt", ["fp8", "mx"])
def test_a_captured_step_of_beam_search(fmt):
    """assign, append, attention, choice, reorder and copies in one graph, everything in place, replayed over page
    boundaries, against the same calls one by one on a second set of buffers."""
    groups, beams, page, hq, hkv, D, vocab = 2, 3, 16, 4, 2, 64, 200
    seqs, max_len, eos, first = groups * beams, 64, 5, 13
    rng = np.random.default_rng(3)
    te = [KR.bf16(rng.standard_normal((vocab, n * D))).to(DEV) for n in (hq, hkv, hkv)]
    head = torch.from_numpy(rng.standard_normal((hq * D, vocab)) * 0.2).float().to(DEV)
    start = rng.integers(8, vocab, (seqs, first))
    cols = max_len // page
    tables = [torch.from_numpy(t).to(DEV) for t in KR_tables(max_len, D)]

    class State:
        def __init__(self):
            z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
            self.cache = empty_cache(seqs * cols + 1, page, hkv, D, fmt)
            self.pool = S.alloc_kv_pool(seqs * cols + 1)
            self.lens, self.held, self.offs = z(seqs), z(seqs), z(seqs + 1)
            self.table, self.own, self.ids = z(seqs, cols), z(seqs, cols), z(seqs, max_len + 1)
            self.scores = torch.zeros((groups, beams), device=DEV) - torch.arange(beams, device=DEV)
            self.done = torch.zeros((groups, beams), dtype=torch.uint8, device=DEV)
            self.parents, self.tokens, self.copies = z(groups, beams), z(groups, beams), z(seqs, 3)
            self.x, self.out = torch.zeros((seqs, vocab), device=DEV), torch.zeros((seqs, hq * D), dtype=torch.bfloat16, device=DEV)
            self.ids[:, :first] = i32(start)
            self.one = i32([first] * seqs)
            req = self.requests(self.one, seqs * first)
            S.sharq_kv_assign(self.pool, req)
            tok = torch.from_numpy(start.reshape(-1)).to(DEV)
            S.sharq_kv_append(None, te[1][tok], te[2][tok], self.cache, req.batch(first), *tables)
            self.one.fill_(1)
            self.tokens.copy_(i32(start[:, -1].reshape(groups, beams)))
            self.req = self.requests(self.one, seqs)
            self.batch = self.req.batch(1)
            need = (S.attention_workspace_bytes(self.cache, self.batch, hq), S.kv_assign_workspace_bytes(self.req),
                    S.beam_workspace_bytes(groups, beams, vocab))
            self.ws = [torch.empty(max(n, 1), dtype=torch.uint8, device=DEV) for n in need]

        def requests(self, add, rows):
            return S.KVRequests(self.lens, add, self.held, self.offs, self.lens, self.table, rows, max_len, page,
                                own_table=self.own)

        def step(self):
            S.sharq_kv_assign(self.pool, self.req, workspace=self.ws[1])
            tok = self.tokens.view(-1)
            q = S.sharq_kv_append(te[0].index_select(0, tok), te[1].index_select(0, tok), te[2].index_select(0, tok),
                                  self.cache, self.batch, *tables)
            S.sharq_attention(q, self.cache, self.batch, out=self.out, workspace=self.ws[0])
            torch.mm(self.out.float(), head, out=self.x)
            S.sharq_beam_select(self.x, self.scores, self.done, eos, self.scores, self.parents, self.tokens, self.done,
                                self.ws[2])
            S.sharq_beam_reorder(self.parents, self.lens, self.table, page, tokens=self.tokens, ids=self.ids,
                                 copies=self.copies)
            S.sharq_kv_copy(self.cache, self.copies)

    a, b = State(), State()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):   # libraries set themselves up outside of the capture
        torch.mm(a.out.float(), head, out=a.x)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        a.step()
    for step in range(40):
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for name in ("lens", "held", "table", "own", "ids", "scores", "parents", "tokens", "done", "copies", "out", "x"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (step, name)
        assert torch.equal(a.pool.count, b.pool.count)
    assert int(a.lens.max()) == first + 40 and int(a.held.max()) == 4
