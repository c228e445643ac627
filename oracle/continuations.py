"""Several continuations of one prompt in numpy and plain Python: selection of beams, forked requests, compaction, copies of pages,
one request, block or token after the other.

The paper scores a tuned model by its answers (Sec. 4.1); beams, samples and the options of a question are this library's reading
of what that takes in serving.
"""
import math

import numpy as np


def beam_select(logits, scores, rows=None, last=None, end_token=-1, lengths=None, power=0.0):
    """-> lists [B][W] of (parent, token, score, length, rank); (-1, -1, -inf, 0, -inf) where there are no more candidates.  Candidates of a beam
    whose ranks round to one number stay in the order of their logits."""
    B, W = scores.shape
    out = []
    for b in range(B):
        found = []
        for w in range(W):
            beam, score = b * W + w, float(scores[b, w])
            length = 0 if lengths is None else int(lengths[b, w])
            if not -math.inf < score < math.inf:
                continue
            if last is not None and int(last[b, w]) == end_token:
                found.append((score / max(length, 1) ** power, beam, 0.0, end_token, score, length))
                continue
            row = beam if rows is None else int(rows[b, w])
            if not 0 <= row < len(logits):
                continue
            x = np.asarray(logits[row], np.float64)
            x = np.where(x < np.inf, x, -np.inf)
            if not (x > -np.inf).any():
                continue
            norm = x.max() + math.log(np.exp(x - x.max()).sum())
            for t in np.argsort(-x, kind="stable")[:W]:
                if x[t] > -np.inf:
                    value = score + (x[t] - norm)
                    found.append((value / max(length + 1, 1) ** power, beam, float(x[t]), int(t), value, length + 1))
        found.sort(key=lambda f: (-f[0], f[1], -f[2], f[3]))
        best = [(beam, t, value, length, rank) for rank, beam, _, t, value, length in found[:W]]
        out.append(best + [(-1, -1, -math.inf, 0, -math.inf)] * (W - len(best)))
    return out


def _held(lens, table, block, n_blocks):
    """Blocks of every request, or None where a length or an id is impossible."""
    held = []
    for n, row in zip(map(int, lens), table):
        if n < 0 or -(-n // block) > len(row):
            return None
        held.append([int(v) for v in row[:-(-n // block)]])
    return held if all(0 <= v < n_blocks for row in held for v in row) else None


def fork_requests(lens, parents, table, free, free_count, block, n_blocks):
    """The new state as a dict, or None when it cannot be served."""
    held = _held(lens, table, block, n_blocks)
    B, width = table.shape
    if held is None or free_count < 0 or any(p >= B for p in parents):
        return None
    stack = [int(v) for v in free[:free_count]]
    kept = {v for r in range(B) if r in set(int(p) for p in parents) for v in held[r]}
    stack += sorted({v for row in held for v in row} - kept)
    if len(stack) > len(free):
        return None
    free = np.array(free)
    free[:len(stack)] = stack
    table_out, lens_out, copies, seen = np.full((B, width), -1, np.int32), [], [], set()
    for r, p in enumerate(map(int, parents)):
        if p < 0:
            lens_out.append(0)
            continue
        n, mine = int(lens[p]), list(held[p])
        if n % block and p in seen:
            if not stack:
                return None
            copies.append((mine[-1], stack[-1], n % block))
            mine[-1] = stack.pop()
        seen.add(p)
        lens_out.append(n)
        table_out[r, :len(mine)] = mine
    return {"table": table_out, "lens": lens_out, "free": free, "free_count": len(stack), "copies": copies}


def compact_blocks(lens, table, block, n_blocks, keep):
    """(new table, free list, copies), or None when more than `keep` blocks are held."""
    held = _held(lens, table, block, n_blocks)
    if held is None:
        return None
    live = sorted({v for row in held for v in row})
    n = len(live)
    if n > keep:
        return None
    holes = [v for v in range(n) if v not in set(live)]
    to = dict(zip((v for v in live if v >= n), holes))
    out = np.full(table.shape, -1, np.int32)
    for r, row in enumerate(held):
        out[r, :len(row)] = [to.get(v, v) for v in row]
    return out, list(range(keep - 1, n - 1, -1)), [(a, b, block) for a, b in to.items()]


def copy_blocks(pages, copies):
    """pages [n_blocks][heads][block][dim], in place."""
    for a, b, n in copies:
        pages[b, :, :n] = pages[a, :, :n]
