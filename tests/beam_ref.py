"""Plain references of the beam search's operators (numpy, 64 bits, loops), written from their definitions."""
from __future__ import annotations

import numpy as np


def ceil_div(a, b):
    return -(-a // b)


def log_sums(x):
    """(x cleaned, log sum exp of every row, how far fp32 exponentials and partial sums of 32 may put it off)."""
    x = np.where(np.isnan(x), -np.inf, np.minimum(x.astype(np.float64), float(np.finfo(np.float32).max)))
    with np.errstate(all="ignore"):
        top = np.maximum(x.max(axis=1, keepdims=True), -float(np.finfo(np.float32).max))
        d = x - top
        w = np.exp(d)
        total = w.sum(axis=1)
        # a term: the difference, its product with log2 e and that constant's rest are off by half a step each, |d| 2^-24; the
        # exponential by 2 steps, 2^-22; a sum of up to 32 of them by 31 half steps
        off = (w * (4 * np.abs(np.where(w > 0, d, 0.0)) * 2.0 ** -24 + 2.0 ** -22 + 31 * 2.0 ** -24)).sum(axis=1) / total
        return x, top[:, 0] + np.log(total), off


def beam_select(x, scores, cu, cu_next, max_next, end):
    """parents, tokens, next_scores, end_scores and bounds of the two kinds of scores, with the entries that are written."""
    x, lse, off = log_sums(x)
    rows, total = x.shape[0], max(int(cu_next[-1]), 0)
    parents, tokens, best = np.full(total, -1), np.full(total, -1), np.full(total, -np.inf)
    ends, tol, end_tol = np.full(rows, -np.inf), np.zeros(total), np.zeros(rows)
    half = 2.0 ** -24
    for s in range(len(cu) - 1):
        found = []
        for r in range(cu[s], cu[s + 1]):
            if np.isfinite(scores[r]):
                t = np.flatnonzero(x[r] > -np.inf)
                found.append((float(scores[r]) + (x[r, t] - lse[r]), np.full(t.size, r), t))
        if not found:
            continue
        y, r, t = (np.concatenate(f) for f in zip(*found))
        # (within a beam by the logits themselves: far from the sum's logarithm 64 bits do not tell their scores apart)
        order = np.lexsort((t, -x[r, t], r, -y))
        y, r, t = y[order], r[order], t[order]
        width = min(cu_next[s + 1] - cu_next[s], max_next)
        first = np.arange(y.size) < width
        for k in np.flatnonzero(first & (t == end)):
            ends[r[k]], end_tol[r[k]] = y[k], off[r[k]] + half * abs(y[k])
        going = np.flatnonzero(t != end)[:width]
        at = cu_next[s] + np.arange(going.size)
        parents[at], tokens[at], best[at], tol[at] = r[going], t[going], y[going], off[r[going]] + half * np.abs(y[going])
    return dict(parents=parents, tokens=tokens, next_scores=best, end_scores=ends, tol=tol, end_tol=end_tol)


def row_blocks(length, held, stride, bs):
    length = max(int(length), 0)
    whole, used = length // bs, ceil_div(length, bs)
    return min(whole, stride), min(used, stride), min(max(used, int(held)), stride)


def fork(parents, lens, held, table, refs, free, begin, bs, table_out):
    n, n_blocks, stride, table_out, after = len(lens), len(refs), table.shape[1], table_out.copy(), refs.copy()
    children = [[j for j, p in enumerate(parents) if p == r] for r in range(n)]
    inside = lambda b: 0 <= b < n_blocks  # noqa: E731
    lens_out, held_out, src, dst, tokens = ([], [], [], [], [])
    for r in range(n):
        whole, _, h = row_blocks(lens[r], held[r], stride, bs)
        for c in range(h):
            more = len(children[r]) - 1 if c < whole else -1 if not children[r] else 0
            if inside(table[r, c]):
                after[table[r, c]] += more
    at = begin
    for j, p in enumerate(parents):
        if not 0 <= p < n:
            lens_out.append(0), held_out.append(0), src.append(-1), dst.append(-1), tokens.append(0)
            continue
        whole, used, h = row_blocks(lens[p], held[p], stride, bs)
        keeps = children[p][0] == j
        h = h if keeps else used
        table_out[j, :h] = table[p, :h]
        made, wanted = -1, not keeps and whole < used
        if wanted:
            if 0 <= at < len(free) and inside(free[at]):
                made = int(free[at])
                after[made] += 1
            at += 1
            table_out[j, whole] = made
        lens_out.append(max(int(lens[p]), 0)), held_out.append(h)
        src.append(int(table[p, whole]) if made >= 0 and inside(table[p, whole]) else -1)
        dst.append(made), tokens.append(int(lens[p]) - whole * bs if made >= 0 else 0)
    return dict(table_out=table_out, lens_out=lens_out, held_out=held_out, refs_after=after, copy_src=src, copy_dst=dst,
                copy_tokens=tokens, blocks_taken=[at])


def free(drop, lens, held, table, refs, bs, taken=(), begin=0, end=0):
    after, lens_after, held_after = refs.copy(), [], []
    for b in taken[max(begin, 0):max(end, 0)]:
        if 0 <= b < len(refs):
            after[b] += 1
    for r in range(len(drop)):
        _, _, h = row_blocks(lens[r], held[r], table.shape[1], bs)
        if drop[r]:
            for b in table[r, :h]:
                if 0 <= b < len(refs):
                    after[b] -= 1
        lens_after.append(0 if drop[r] else int(lens[r])), held_after.append(0 if drop[r] else h)
    ids = np.flatnonzero(after <= 0)
    return dict(refs_after=after, free_blocks=np.concatenate([ids, np.full(len(refs) - len(ids), -1)]), n_free=[len(ids)],
                lens_after=lens_after, held_after=held_after)


def compact(refs, n_keep, lens, held, table, bs, n_pairs, table_out):
    n, table_out, after = len(refs), table_out.copy(), refs.copy()
    used = [b for b in range(n) if refs[b] > 0]
    keep = len(used) if n_keep < 0 else min(n_keep, n)
    leave, take = [b for b in used if b >= keep], [b for b in range(keep) if refs[b] <= 0]
    moves = list(zip(leave, take))[:n_pairs]
    where = np.arange(n)
    for a, b in moves:
        where[a], after[b], after[a] = b, refs[a], 0
    for r in range(len(lens)):
        _, _, h = row_blocks(lens[r], held[r], table.shape[1], bs)
        for c in range(h):
            b = table[r, c]
            table_out[r, c] = where[b] if 0 <= b < n else b
    pad = lambda v: v + [-1] * (n_pairs - len(v))  # noqa: E731
    return dict(table_out=table_out, refs_after=after, block_map=where, copy_src=pad([a for a, _ in moves]),
                copy_dst=pad([b for _, b in moves]), counts=[len(used), len(moves), len(leave) - len(moves)])


def shared_pages(rs, sessions, beams, bs, longest, n_blocks, ahead=2):
    """Rows whose sessions share their first blocks: (lens, held, table, refs, ids that nobody holds), all consistent."""
    order, at, lens, held, rows = list(rs.permutation(n_blocks)), 0, [], [], []
    for _ in range(sessions):
        length = int(rs.randint(0, longest + 1))
        first = None
        for _ in range(beams):
            whole, used, _ = row_blocks(length, 0, 1 << 30, bs)
            shared = int(rs.randint(0, whole + 1)) if first is not None else 0
            h = used + int(rs.randint(0, ahead + 1))
            ids = (first[:shared] if shared else []) + order[at:at + h - shared]
            at += h - shared
            first = first or ids
            lens.append(length), held.append(h), rows.append(ids)
    assert at <= n_blocks, (at, n_blocks)
    table = np.full((len(rows), max(held) + 2), -1, np.int32)
    for r, ids in enumerate(rows):
        table[r, :len(ids)] = ids
    refs = np.bincount(table[table >= 0], minlength=n_blocks).astype(np.int32)
    return np.array(lens, np.int32), np.array(held, np.int32), table, refs, np.array(order[at:], np.int32)
