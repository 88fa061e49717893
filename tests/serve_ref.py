"""What stands around the paged cache, on the CPU and from the definitions: tables from request lengths, beam search's
choice, the reordering behind it.  Without the library's code."""

import numpy as np


def assign(free, count, keep, add, held, table, rows, max_len, page, own=None, pages=None):
    """Lists and arrays are changed in place.  Returns a dict of the outputs; of rows behind the last sequence None."""
    pages = len(free) if pages is None else pages
    seqs, cols = len(keep), -(-max_len // page)
    clip = lambda v, lo, hi: max(lo, min(int(v), hi))  # noqa: E731
    count, at = clip(count, 0, pages), 0
    offs, lens, need, before = [0], [], [], []
    for s in range(seqs):
        k = clip(keep[s], 0, max_len)
        n = min(clip(add[s], 0, max_len - k), rows - at)
        at += n
        offs.append(at), lens.append(k + n), need.append(-(-(k + n) // page)), before.append(clip(held[s], 0, cols))
    source = table if own is None else own
    for s in range(seqs):
        for c in range(need[s], before[s]):
            if 0 <= source[s][c] < pages and count < pages:
                free[count] = source[s][c]
                count += 1
    missing = 0
    for s in range(seqs):
        for c in range(before[s], need[s]):
            if count > 0:
                count -= 1
                p = free[count]
            else:
                p, missing = -1, missing + 1
            table[s][c] = p
            if own is not None:
                own[s][c] = p
    row_seq, positions, slots = [None] * rows, [None] * rows, [None] * rows
    for s in range(seqs):
        for r in range(offs[s], offs[s + 1]):
            p = lens[s] - (offs[s + 1] - r)
            pg = table[s][p // page]
            row_seq[r], positions[r], slots[r] = s, p, pg * page + p % page if 0 <= pg < pages else -1
    return dict(row_offsets=offs, lens=lens, held=need, count=count, missing=missing, row_seq=row_seq,
                positions=positions, slots=slots)


def log_probabilities(x):
    """x [vocab] float64 -> x - ln sum e^x, NaN where it has none."""
    with np.errstate(all="ignore"):
        top = x.max() if len(x) else -np.inf
        return x - (top + np.log(np.exp(x - top).sum()))


def candidates(x, scores, done, eos, most=None):
    """x [beams, vocab], scores [beams] -> [(score, beam, token)], the best first, ties by the lower beam, within a beam by
    the logits and the lower token; of each beam the first `most`."""
    out = []
    for b in range(len(scores)):
        if not np.isfinite(scores[b]):
            continue
        if done is not None and done[b]:
            out.append((float(scores[b]), b, eos))
            continue
        with np.errstate(all="ignore"):
            t = np.float64(scores[b]) + log_probabilities(x[b])
        at = np.nonzero(t > -np.inf)[0]
        if most is not None and len(at) > 4 * most:      # those that reach the `most`-th largest
            at = at[x[b][at] >= np.partition(x[b][at], len(at) - most)[len(at) - most]]
        at = at[np.lexsort((at, -x[b][at]))][:most]
        out += [(float(t[v]), b, int(v)) for v in at]
    return sorted(out, key=lambda c: (-c[0], c[1]))


def reorder(parents, length, page, table, ids=None, tokens=None):
    """One group: parents [beams], table [beams][cols], ids [beams][n].  Returns (table, copies, ids), new ones."""
    beams = len(parents)
    parents = [max(0, min(int(p), beams - 1)) for p in parents]
    whole, part = length // page, length % page
    new = [list(r) for r in table]
    copies = [(-1, -1, -1)] * beams
    idle = [p for p in range(beams) if p not in parents]
    seen = set()
    for i, p in enumerate(parents):
        new[i][:whole] = list(table[p][:whole])
        taken = p
        if p in seen:
            taken = idle.pop(0)
            if part and whole < len(table[0]):
                copies[i] = (table[p][whole], table[taken][whole], part)
        seen.add(p)
        if part and whole < len(table[0]):
            new[i][whole] = table[taken][whole]
    out = None
    if ids is not None:
        out = [list(r) for r in ids]
        for i, p in enumerate(parents):
            out[i][:length] = list(ids[p][:length])
            if length < len(out[i]):
                out[i][length] = tokens[i]
    return new, copies, out
