"""Tables and slot maps from request lengths on the GPU, against the definition: whole numbers, all of them equal."""

import numpy as np
import pytest
import torch

import serve_ref as R
from paper_2606_26587_amd import sharq as S

pytestmark = pytest.mark.gpu
DEV = "cuda"
LEFT = -77


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def make(seqs, max_len, page, rng, pages=None, ended=0.2, new=0.2, most=40):
    """Random requests over disjoint pages: (free, count, keep, add, held, table)."""
    cols = -(-max_len // page)
    lens = rng.integers(0, max_len + 1, seqs)
    held = -(-lens // page)
    total = int(held.sum())
    pages = total + seqs * 2 + 5 if pages is None else pages
    ids = rng.permutation(max(pages, total))
    table = np.full((seqs, cols + 2), LEFT)
    at = 0
    for s in range(seqs):
        table[s, :held[s]] = ids[at:at + held[s]]
        at += held[s]
    free = np.full(pages, LEFT)
    count = max(0, pages - total)
    free[:count] = ids[total:total + count]
    u = rng.random(seqs)
    keep = np.where(u < ended, 0, np.where(u < ended + new, rng.integers(0, lens + 1), lens))
    add = np.where(u < ended / 2, 0, np.where(rng.random(seqs) < 0.3, rng.integers(0, most + 1, seqs), 1))
    return free, count, keep, add, held, table


def run_and_check(free, count, keep, add, held, table, rows, max_len, page, own=None, in_place=False, ld_extra=3):
    seqs, width = table.shape
    t_free, t_count = i32(free), i32([count])
    wide = torch.full((seqs, width + ld_extra), LEFT, dtype=torch.int32, device=DEV)
    t_table = wide[:, :width]
    t_table.copy_(i32(table))
    t_own = None
    if own is not None:
        t_own = torch.full_like(wide, LEFT)[:, :width]
        t_own.copy_(i32(own))
    t_keep, t_add, t_held = i32(keep), i32(add), i32(held)
    blank = lambda n: torch.full((n,), LEFT, dtype=torch.int32, device=DEV)  # noqa: E731
    out = {n: blank(rows) for n in ("row_seq", "positions", "slots")}
    offs, missing = blank(seqs + 1), blank(1)
    lens = t_keep if in_place else blank(seqs)
    held_out = None if in_place else blank(seqs)
    count_out = None if in_place else blank(1)
    pool = S.KVPool(t_free, t_count, count_out)
    req = S.KVRequests(t_keep, t_add, t_held, offs, lens, t_table, rows, max_len, page, held_out=held_out,
                       own_table=t_own, missing=missing, **out)
    S.sharq_kv_assign(pool, req)
    torch.cuda.synchronize()
    free, table = list(free), np.array(table)
    own = None if own is None else np.array(own)
    want = R.assign(free, count, keep, add, held, table, rows, max_len, page, own)
    host = lambda t: t.cpu().numpy()  # noqa: E731
    assert list(host(offs)) == want["row_offsets"]
    assert list(host(lens)) == want["lens"]
    assert list(host(t_held if in_place else held_out)) == want["held"]
    assert int(t_count if in_place else count_out) == want["count"]
    assert int(missing) == want["missing"]
    assert np.array_equal(host(t_table), table) and (host(wide)[:, width:] == LEFT).all()
    assert own is None or np.array_equal(host(t_own), own)
    assert list(host(t_free)[:want["count"]]) == [int(p) for p in free[:want["count"]]]
    for n in ("row_seq", "positions", "slots"):
        assert list(host(out[n])) == [LEFT if v is None else v for v in want[n]], n
    if not in_place:
        assert np.array_equal(host(t_keep), keep) and np.array_equal(host(t_held), held) and int(t_count) == count
    return req, want


@pytest.mark.parametrize("seqs,max_len,page,pad", [
    (1, 1, 16, 0), (1, 100, 16, 3), (3, 40, 16, 0), (64, 300, 32, 1), (65, 17, 16, 9), (257, 500, 64, 0),
    (1000, 90, 16, 5), (1025, 33, 16, 2), (2048, 20, 16, 0),       # one workgroup
    (2049, 20, 16, 3), (5000, 100, 16, 50),                        # two launches
])
@pytest.mark.parametrize("in_place", [False, True])
def test_random_requests(seqs, max_len, page, pad, in_place):
    rng = np.random.default_rng(seqs)
    args = make(seqs, max_len, page, rng)
    rows = int(np.minimum(args[3], max_len - args[2]).sum()) + pad
    run_and_check(*args, rows, max_len, page, in_place=in_place)


@pytest.mark.parametrize("adds", [[9000], [0, 0, 8192, 0], [1] * 100 + [9000] + [0] * 70 + [1] * 100,
                                  [0] * 200 + [5000] + [0] * 200 + [7, 6000] + [0] * 64,
                                  [20000] + [0] * 128])
def test_long_prompts_and_empty_requests(adds):
    """More rows than one workgroup takes; rows of a wavefront around runs of empty sequences."""
    rng = np.random.default_rng(len(adds))
    seqs = len(adds)
    cols = -(-21000 // 64)
    pages = sum(-(-a // 64) for a in adds) + 3
    free = rng.permutation(pages)
    table = np.full((seqs, cols), LEFT)
    run_and_check(free, pages, [0] * seqs, adds, [0] * seqs, table, sum(adds) + 70, 21000, 64)


def test_few_rows_between_many_empty_sequences():
    adds = np.zeros(3000, int)
    adds[[0, 1, 700, 701, 1500, 2999]] = 1
    run_and_check(np.arange(50), 50, np.zeros(3000, int), adds, np.zeros(3000, int), np.full((3000, 4), LEFT), 9000, 64, 16)


@pytest.mark.parametrize("seqs,rows", [(5, 100), (2500, 9000)])
@pytest.mark.parametrize("pages", [0, 1, 7, 30])
def test_pages_run_out(seqs, rows, pages):
    """Some columns get none; of the rows there the slot is -1, and the count says how many pages were missing."""
    rng = np.random.default_rng(pages)
    adds = rng.integers(0, 40, seqs)
    table = np.full((seqs, 3), LEFT)
    _, want = run_and_check(rng.permutation(pages), pages, np.zeros(seqs, int), adds, np.zeros(seqs, int), table, rows, 40, 16)
    assert (want["missing"] > 0) == (sum(-(-int(a) // 16) for a in adds) > pages)


@pytest.mark.parametrize("seqs", [40, 3000])
def test_pages_that_come_back_are_given_out_again(seqs):
    """Nothing is free before the call: what the ended requests held goes to the new ones."""
    keep, add, held = np.zeros(seqs, int), np.zeros(seqs, int), np.zeros(seqs, int)
    held[::2], add[1::2] = 2, 30
    table = np.full((seqs, 2), LEFT)
    table[::2] = np.arange(seqs).reshape(-1, 2)
    free = np.full(seqs, LEFT)
    _, want = run_and_check(free, 0, keep, add, held, table, 15 * seqs + 1, 32, 16)
    assert want["missing"] == 0 and want["count"] == 0


def test_rows_run_out():
    """Requests beyond the call's rows are cut: their lengths say how much came in."""
    for rows in (0, 1, 10, 37, 100):
        run_and_check(np.arange(60), 60, [3, 0, 20, 5], [10, 30, 8, 50], [1, 0, 2, 1],
                      np.array([[50, LEFT, LEFT, LEFT]] + [[LEFT] * 4] + [[51, 52, LEFT, LEFT]] + [[53, LEFT, LEFT, LEFT]]),
                      rows, 64, 16)


def test_values_outside_their_range():
    """Negative and overlong lengths, columns and entries count as the nearest in range, and touch nothing else."""
    big = 2 ** 31 - 1
    for count in (-5, 3, 1000):
        run_and_check(np.arange(8), count, [-4, big, 40, 3, 0], [5, big, -1, big, 0], [-1, 2, big, 1, big],
                      np.array([[LEFT] * 6, [1, 2, LEFT, LEFT, LEFT, LEFT], [3, 4, 99, -1, 5, 6],
                                [7, LEFT, LEFT, LEFT, LEFT, LEFT], [2 ** 31 - 1, -2 ** 31, 8, 0, 1, 2]]), 70, 64, 16)


def test_sequences_with_pages_of_others():
    """Beams: their tables name shared pages, own_table those that they hold themselves; only these go back."""
    table = np.array([[5, 6, 1, LEFT], [5, 6, 2, LEFT], [5, 6, 3, LEFT], [9, LEFT, LEFT, LEFT]])
    own = np.array([[5, 6, 1, LEFT], [-1, -1, 2, LEFT], [-1, -1, 3, LEFT], [9, LEFT, LEFT, LEFT]])
    free = np.array([0, 4, 7, 8, 10, 11] + [LEFT] * 6)
    run_and_check(free, 6, [48, 48, 48, 10], [1, 1, 1, 1], [3, 3, 3, 1], table, 4, 64, 16, own=own)
    run_and_check(free, 6, [0, 0, 0, 10], [0, 0, 0, 1], [3, 3, 3, 1], table, 4, 64, 16, own=own)


def test_no_sequences_and_no_pages():
    one = lambda: i32([])  # noqa: E731
    offs, count = i32([LEFT]), i32([3])
    req = S.KVRequests(one(), one(), one(), offs, one(), torch.empty((0, 4), dtype=torch.int32, device=DEV), 20000, 64, 16)
    S.sharq_kv_assign(S.KVPool(i32([4, 5, 6, 0]), count), req)
    assert int(offs) == 0 and int(count) == 3
    run_and_check(np.array([], int), 0, [0, 0], [0, 5], [0, 0], np.full((2, 1), LEFT), 5, 16, 16)


@pytest.mark.parametrize("rows,seqs", [(40, 12), (9000, 12)])
def test_captured_steps(rows, seqs):
    """A decode loop in a graph: lengths, columns and the pool are carried on in place."""
    rng = np.random.default_rng(1)
    pages, page, max_len = 200, 16, 300
    free = rng.permutation(pages)
    lens, held = i32([0] * seqs), i32([0] * seqs)
    add = i32([0] * seqs)
    offs, slots = i32([0] * (seqs + 1)), i32([LEFT] * rows)
    table = torch.full((seqs, 19), LEFT, dtype=torch.int32, device=DEV)
    pool = S.KVPool(i32(free), i32([pages]))
    req = S.KVRequests(lens, add, held, offs, lens, table, rows, max_len, page, slots=slots)
    ws = torch.empty(S.kv_assign_workspace_bytes(req), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        S.sharq_kv_assign(pool, req, workspace=ws)
    state = dict(free=list(free), count=pages, lens=[0] * seqs, held=[0] * seqs, table=np.full((seqs, 19), LEFT))
    for step in range(12):
        n = rng.integers(0, 4, seqs) if step else rng.integers(1, 60 if rows > 100 else 4, seqs)
        ended = rng.random(seqs) < (0.2 if step % 3 == 2 else 0)
        keep = np.where(ended, 0, state["lens"])
        add.copy_(i32(n))
        lens.copy_(i32(keep))
        graph.replay()
        torch.cuda.synchronize()
        want = R.assign(state["free"], state["count"], keep, n, state["held"], state["table"], rows, max_len, page)
        state.update(count=want["count"], lens=want["lens"], held=want["held"])
        assert list(lens.cpu().numpy()) == want["lens"] and list(held.cpu().numpy()) == want["held"]
        assert np.array_equal(table.cpu().numpy(), state["table"])
        total = want["row_offsets"][-1]
        assert list(slots.cpu().numpy()[:total]) == want["slots"][:total]
        assert int(pool.count) == want["count"]
        in_use = [p for s in range(seqs) for p in state["table"][s][:want["held"][s]]]
        assert len(set(in_use)) == len(in_use) == pages - want["count"]


def test_on_a_stream_of_its_own():
    rng = np.random.default_rng(4)
    free, count, keep, add, held, table = make(100, 200, 16, rng)
    side = torch.cuda.Stream()
    offs, lens = i32([0] * 101), i32([0] * 100)
    pool = S.KVPool(i32(free), i32([count]))
    req = S.KVRequests(i32(keep), i32(add), i32(held), offs, lens, i32(table), 5000, 200, 16)
    side.wait_stream(torch.cuda.current_stream())
    S.sharq_kv_assign(pool, req, stream=side)
    side.synchronize()
    want = R.assign(list(free), count, keep, add, held, np.array(table), 5000, 200, 16)
    assert list(offs.cpu().numpy()) == want["row_offsets"] and list(lens.cpu().numpy()) == want["lens"]
