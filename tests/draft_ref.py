"""Plain references of the speculative step's operators (numpy, 64 bits, loops), written from their definitions."""
from __future__ import annotations

import numpy as np


def ceil_div(a, b):
    return -(-a // b)


def build_tables(prefix, new, table, free, block_size, n_blocks, total, held=None, free_begin=0):
    table = table.copy()
    cu, at = [0], free_begin
    slots, positions, held_after = np.full(total, -1, np.int64), np.full(total, -1, np.int32), []
    stride, t = table.shape[1], 0
    for s, (P, N) in enumerate(zip(np.maximum(prefix, 0), np.maximum(new, 0))):
        H = max(ceil_div(P, block_size), 0 if held is None else held[s])
        need = max(ceil_div(P + N, block_size) - H, 0)
        ids = [int(free[at + j]) if 0 <= at + j < len(free) else -1 for j in range(need)]
        for i in range(N):
            if t < total:
                b, place = divmod(P + i, block_size)
                if b >= H and place == 0 and b < stride:
                    table[s, b] = ids[b - H]
                block = -1 if b >= stride else (ids[b - H] if b >= H else table[s, b])
                if 0 <= block < n_blocks:
                    slots[t] = int(block) * block_size + place
                positions[t] = P + i
            t += 1
        at += need
        held_after.append(H + need)
        cu.append(cu[-1] + N)
    return dict(table=table, cu=np.array(cu, np.int32), offsets=np.array(cu, np.int64), slots=slots, positions=positions,
                taken=np.array([at], np.int32), held_after=np.array(held_after, np.int32))


def ancestors(parents):
    """sees[i][j]: node j is node i or an ancestor of it (one session)."""
    n = len(parents)
    sees = np.zeros((n, n), bool)
    for i in range(n):
        j = i
        while True:
            sees[i, j] = True
            if not 0 <= parents[j] < j:
                break
            j = parents[j]
    return sees


def pack_bits(rows, words):
    """Packed words of a list of boolean [N_s][N_s] masks, as int64 [T][words]."""
    total = sum(len(r) for r in rows)
    bits = np.zeros((total, words * 64), np.uint8)
    t = 0
    for r in rows:
        k = min(r.shape[1], words * 64) if len(r) else 0
        bits[t:t + len(r), :k] = r[:, :k]
        t += len(r)
    return np.packbits(bits, axis=1, bitorder="little").view(np.int64).reshape(total, words)


def accept(draft, parents, target):
    """Accepted nodes of one session's tree, in order."""
    if len(draft) == 0:
        return []
    path = [0]
    while True:
        children = [j for j in range(path[-1] + 1, len(draft)) if parents[j] == path[-1] and draft[j] == target[path[-1]]]
        if not children:
            return path
        path.append(children[0])


def tree_attn(k_pool, v_pool, q, k_new, v_new, sees, cu, prefix, table, scale):
    """(out, bound) in 64 bits: the result, and sum_j p_j |v_j| with the largest |score| sum of the row, from which tests derive
    how far a computation in fewer bits may be off.  Pools [n_blocks][bs][H_kv][d] of one layer; sees: one mask per session."""
    n_blocks, bs, hkv, d = k_pool.shape
    T, hq, _ = q.shape
    g = hq // hkv
    out, weight, spread = np.zeros((T, hq, d)), np.zeros((T, hq, d)), np.zeros((T, hq))
    f = lambda a: a.astype(np.float64)  # noqa: E731
    with np.errstate(all="ignore"):
        for s, P in enumerate(prefix):
            a, b = cu[s], cu[s + 1]
            if a == b:
                continue
            ids = np.array([table[s, j // bs] for j in range(P)], dtype=np.int64)
            inside = (ids >= 0) & (ids < n_blocks)
            for h in range(hkv):
                k, v = (np.concatenate([np.where(inside[:, None], f(pool[np.where(inside, ids, 0), np.arange(P) % bs, h]), 0.0),
                                        f(new[a:b, h])]) for pool, new in ((k_pool, k_new), (v_pool, v_new)))
                for i in range(b - a):
                    seen = np.concatenate([np.ones(P, bool), sees[s][i]])
                    if not seen.any():
                        continue
                    ks, vs = k[seen], v[seen]
                    for hh in range(h * g, (h + 1) * g):
                        qi = f(q[a + i, hh])
                        x = scale * (ks @ qi)
                        p = np.exp(x - x.max())
                        p /= p.sum()
                        out[a + i, hh] = (p[:, None] * vs).sum(axis=0)
                        weight[a + i, hh] = (p[:, None] * np.abs(vs)).sum(axis=0)
                        spread[a + i, hh] = scale * (np.abs(ks) @ np.abs(qi)).max()
    return out, weight, spread
