"""The operators of beam search over the paged cache, as cases that can be timed and compared.

A step of beam search scores every beam's next tokens, keeps each session's best continuations and gives them their beams' cached
tokens: rows of the block table that share all full blocks, with copies of the blocks that are still being filled.  Blocks that no
row holds any more become free, and the blocks of a pool that has to shrink move together.  Five operators, each in its plain form
(elementary torch operations) and through the package:

  beam     `beam_select`: the best continuations of every session over its beams and the vocabulary
  fork     `kv_fork`: table rows, reference counts and block copies for rows that continue other rows
  copy     `kv_copy_blocks`: blocks of all layers to other places of the pools
  free     `kv_free`: references of dropped rows given back, the list of free blocks
  compact  `kv_compact`: which blocks move to empty a pool's end, tables and counts after the move

A case is a dict of plain values.  Its lengths follow from the case alone (`lens`, a seed, and the ranges named in it); logits,
block ids, parents and values follow from the seed that `prepare` is given.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"

# The pools of the 8B shape: 32 layers, 8 kv-heads, head_dim 128, bf16, blocks of 16 tokens.
_8B = dict(op="copy", dtype="bf16", layers=32, hkv=8, d=128, bs=16)
# 64 sessions of eight beams over prompts of up to 8192 tokens, in a pool of 131072 such blocks (256 GiB).
_SERVER = dict(bs=16, sessions=64, beams=8, p_lo=512, p_hi=8192, g_hi=400, blocks=131072)


def listed():
    return [
        # One user, four beams of a small vocabulary in fp32: latency only.
        dict(op="beam", name="beam_one_user", dtype="fp32", sessions=1, b_lo=4, b_hi=4, w_hi=4, vocab=32000, masked=0, end=1, lens=1),
        # Sessions of different widths, an odd vocabulary, most tokens ruled out by a grammar, some beams ended.
        dict(op="beam", name="beam_odd_masked", dtype="fp32", sessions=7, b_lo=1, b_hi=24, w_hi=24, vocab=50001, masked=90, end=1,
             lens=2),
        # A full server: 512 beams over a large vocabulary.
        dict(op="beam", name="beam_server", dtype="bf16", sessions=64, b_lo=8, b_hi=8, w_hi=8, vocab=128256, masked=0, end=1, lens=3),
        # The beams of one user's step, 3000 tokens long.
        dict(op="fork", name="fork_one_user", bs=16, sessions=1, beams=4, p_lo=3000, p_hi=3000, g_hi=60, blocks=1024, out=4, short=0,
             lens=4),
        # The same for a full server.
        dict(_SERVER, op="fork", name="fork_server", out=8, short=0, lens=5),
        # What a fork copies for one user of a small fp32 model with odd blocks.
        dict(op="copy", name="copy_small_fp32", dtype="fp32", layers=4, hkv=2, d=64, bs=24, pairs=5, whole=0, skip=40, lens=6),
        # What a fork copies for a full server: the filled slots of about half the rows' last blocks.
        dict(_8B, name="copy_fork_server", pairs=512, whole=0, skip=45, lens=7),
        # The moves of a compaction: whole blocks.
        dict(_8B, name="copy_moves", pairs=448, whole=1, skip=0, lens=8),
        # One user of a small pool is done.
        dict(op="free", name="free_one_user", bs=16, sessions=2, beams=4, p_lo=1000, p_hi=3000, g_hi=60, blocks=1024, drop=50, lens=9),
        # A quarter of a full server's sessions are done.
        dict(_SERVER, op="free", name="free_server", drop=25, lens=10),
        # A small pool is packed together.
        dict(op="compact", name="compact_small", bs=16, sessions=4, beams=2, p_lo=200, p_hi=3000, g_hi=60, blocks=2048, keep=0, lens=11),
        # A full server gives back the last quarter of its pool.
        dict(_SERVER, op="compact", name="compact_server", keep=75, lens=12),
    ]


# ------------------------------------------------------------------------------------------------------------------
# lengths and the work of a case
# ------------------------------------------------------------------------------------------------------------------
def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def _starts(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int64)


def _ceil(a, b):
    return -(-a // b)


def _widths(case):
    """(beams, continuations that are asked for) of every session."""
    rng = random.Random(case["lens"])
    beams = [rng.randint(case["b_lo"], case["b_hi"]) for _ in range(case["sessions"])]
    return beams, [b if rng.random() < 0.7 else rng.randint(1, case["w_hi"]) for b in beams]


def _dead(case):
    """Beams that have ended: about one in eight where there are several, for cases with ruled-out tokens."""
    rng = random.Random(case["lens"] + 1)
    return [case["masked"] > 0 and b > 1 and rng.random() < 0.125 for b in _widths(case)[0] for _ in range(b)]


def _row_lens(case):
    """(cached tokens of every row, tokens at its front that are the first row's of its session)."""
    rng = random.Random(case["lens"])
    lens, common = [], []
    for _ in range(case["sessions"]):
        p, g = rng.randint(case["p_lo"], case["p_hi"]), rng.randint(0, case["g_hi"])
        lens += [p + g] * case["beams"]
        common += [0] + [p + rng.randint(0, g) for _ in range(case["beams"] - 1)]
    return np.array(lens), np.array(common)


def _ahead(case):
    """Blocks that a row holds behind the ones in use: none or one."""
    rng = random.Random(case["lens"] + 2)
    return np.array([rng.choice([0, 0, 1]) for _ in range(case["sessions"] * case["beams"])])


def _own_blocks(case):
    """(blocks held, blocks shared with the session's first row, blocks of the row alone) of every row."""
    lens, common = _row_lens(case)
    held, shared = _ceil(lens, case["bs"]) + _ahead(case), common // case["bs"]
    return held, shared, held - shared


def _n_blocks(case):
    return max(case["blocks"], int(_own_blocks(case)[2].sum()) + 8)


def _dropped(case):
    rng = random.Random(case["lens"] + 3)
    gone = [rng.random() * 100 < case["drop"] for _ in range(case["sessions"])]
    return np.repeat(np.array(gone, dtype=np.int32), case["beams"])


def _n_keep(case):
    """Blocks of the pool that stay: a share of them, or (-1) as many as are in use."""
    return _n_blocks(case) * case["keep"] // 100 if case["keep"] else -1


def _n_moves(case):
    """Entries of the lists of moves: as many as there can be, half of the pool at most."""
    n, keep = _n_blocks(case), _n_keep(case)
    return min(int(_own_blocks(case)[2].sum()), n // 2 if keep < 0 else n - keep)


def _copied(case):
    """Tokens of every pair of blocks, 0 for a pair that is left out."""
    rng = random.Random(case["lens"])
    return [0 if rng.random() * 100 < case["skip"] else case["bs"] if case["whole"] else rng.randint(1, case["bs"])
            for _ in range(case["pairs"])]


def work(case):
    op = case["op"]
    if op == "beam":
        (beams, wide), rows = _widths(case), len(_dead(case))
        return {"bytes": (rows - sum(_dead(case))) * case["vocab"] * _elem(case) + 8 * rows + 8 * (len(beams) + 1) + 12 * sum(wide),
                "flops": 4.0 * (rows - sum(_dead(case))) * case["vocab"]}
    if op == "copy":
        return {"bytes": 4 * sum(_copied(case)) * case["layers"] * case["hkv"] * case["d"] * _elem(case) + 12 * case["pairs"], "flops": 0}
    n, held = _n_blocks(case), _own_blocks(case)[0]
    if op == "fork":
        # (as if every row had one child: tables read and written, counts before and after, a few words for each row)
        per_session = held.reshape(case["sessions"], -1).mean(axis=1).sum()
        return {"bytes": int(8 * per_session * case["out"]) + 8 * n + 8 * len(held) + 24 * case["sessions"] * case["out"], "flops": 0}
    if op == "free":
        return {"bytes": 4 * int((held * _dropped(case)).sum()) + 12 * n + 20 * len(held), "flops": 0}
    return {"bytes": 12 * n + 8 * _n_moves(case) + 8 * int(held.sum()) + 8 * len(held), "flops": 0}


# ------------------------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------------------------
def _i32(values):
    return torch.from_numpy(np.ascontiguousarray(values, dtype=np.int32)).to(DEVICE)


def _e32(n):
    return torch.zeros(n, dtype=torch.int32, device=DEVICE)


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _prepare_beam(case, seed):
    (beams, wide), dead, g = _widths(case), np.array(_dead(case)), _generator(seed)
    rows, rs = len(dead), np.random.RandomState(seed % (1 << 31))
    logits = torch.empty((rows, case["vocab"]), dtype=_dtype(case), device=DEVICE).normal_(0.0, 3.0, generator=g)
    if case["masked"]:
        ruled_out = torch.empty((rows, case["vocab"]), device=DEVICE).uniform_(0.0, 100.0, generator=g) < case["masked"]
        logits.masked_fill_(ruled_out, -math.inf)
    scores = rs.uniform(-12.0, -2.0, size=rows).astype(np.float32)
    scores[dead] = -math.inf
    total = sum(wide)
    return dict(op="beam", logits=logits, scores=torch.from_numpy(scores).to(DEVICE), cu=_i32(_starts(beams)), cu_next=_i32(_starts(wide)),
                max_next=max(wide), end=rs.randint(case["vocab"]) if case["end"] else -1, parents=_e32(total), tokens=_e32(total),
                next_scores=torch.zeros(total, device=DEVICE), end_scores=torch.zeros(rows, device=DEVICE))


def _pages(case, seed):
    """A pool whose rows of a session share the blocks of their common tokens: what a server keeps of it, on the device."""
    rs = np.random.RandomState(seed % (1 << 31))
    lens, _ = _row_lens(case)
    held, shared, alone = _own_blocks(case)
    n, rows = _n_blocks(case), len(held)
    order = rs.permutation(n)
    at, first = _starts(alone)[:-1, None], (np.arange(rows) // case["beams"]) * case["beams"]
    cols = np.arange(int(held.max()) + 3)[None, :]
    which = np.where(cols < shared[:, None], at[first] + cols, at + cols - shared[:, None])
    table = np.where(cols < held[:, None], order[np.minimum(which, n - 1)], -1)
    refs = np.bincount(table[table >= 0], minlength=n)
    return rs, dict(lens=_i32(lens), held=_i32(held), table=_i32(table), refs=_i32(refs), bs=case["bs"],
                    refs_after=_e32(n)), order[int(alone.sum()):]


def _prepare_fork(case, seed):
    rs, st, free = _pages(case, seed)
    out, beams = case["out"] * case["sessions"], case["beams"]
    # better beams have more children; one continuation in 32 has ended
    pick = np.floor(beams * rs.random_sample(out) ** 1.5).astype(np.int64)
    parents = np.where(rs.random_sample(out) < 1 / 32, -1, np.arange(out) // case["out"] * beams + pick)
    # (a list that ends too early by `short` blocks of what the widest step needs)
    begin = int(rs.randint(0, 3))
    free = free[:max(1, min(len(free), out) - case["short"])] if case["short"] else free
    st.update(op="fork", parents=_i32(parents), free=_i32(free), begin=_i32([begin]), taken=_e32(1), lens_out=_e32(out),
              held_out=_e32(out), table_out=torch.full((out, st["table"].shape[1]), -1, dtype=torch.int32, device=DEVICE),
              copy_src=_e32(out), copy_dst=_e32(out), copy_tokens=_e32(out))
    return st


def _prepare_free(case, seed):
    rs, st, _ = _pages(case, seed)
    n, rows = st["refs"].numel(), st["lens"].numel()
    st.update(op="free", drop=_i32(_dropped(case)), free=_e32(n), n_free=_e32(1), lens_after=_e32(rows), held_after=_e32(rows))
    return st


def _prepare_compact(case, seed):
    rs, st, _ = _pages(case, seed)
    moves = _n_moves(case)
    st.update(op="compact", n_keep=_n_keep(case), table_out=st["table"].clone(), map=_e32(st["refs"].numel()), copy_src=_e32(moves),
              copy_dst=_e32(moves), counts=_e32(3))
    return st


def _prepare_copy(case, seed):
    rs, g, tokens = np.random.RandomState(seed % (1 << 31)), _generator(seed), np.array(_copied(case))
    n = 2 * case["pairs"] + 3
    ids = rs.permutation(n)
    src, dst = (np.where(tokens > 0, ids[k * case["pairs"]:(k + 1) * case["pairs"]], -1) for k in range(2))
    pool = (case["layers"], n, case["bs"], case["hkv"], case["d"])
    make = lambda: torch.empty(pool, dtype=_dtype(case), device=DEVICE).normal_(0.0, 1.0, generator=g)  # noqa: E731
    return dict(op="copy", k_pool=make(), v_pool=make(), src=_i32(src), dst=_i32(dst), tokens=None if case["whole"] else _i32(tokens))


_PREPARE = {"beam": _prepare_beam, "fork": _prepare_fork, "copy": _prepare_copy, "free": _prepare_free, "compact": _prepare_compact}


def prepare(case, seed):
    return _PREPARE[case["op"]](case, seed)


# ------------------------------------------------------------------------------------------------------------------
# the plain forms
# ------------------------------------------------------------------------------------------------------------------
def _plain_beam(st):
    """In 64 bits: the order of scores that are nearly equal is part of the answer."""
    x, cu, cu_next = st["logits"].double(), st["cu"].long(), st["cu_next"].long()
    rows, vocab = x.shape
    top = x.amax(dim=1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    log_sum = torch.log(torch.exp(x - top).sum(dim=1, keepdim=True)) + top
    scores = st["scores"].double()[:, None] + (x - log_sum)
    scores = torch.where(torch.isnan(scores), torch.full_like(scores, -math.inf), scores)  # (a row without any token)
    row = torch.arange(rows, device=DEVICE)
    session = torch.searchsorted(cu[1:], row, right=True)
    width = cu_next[1:] - cu_next[:-1]
    # a row gives its session at most as many as are wanted there, and one that ends: what equals the last of them is looked at too
    least = torch.topk(scores, min(st["max_next"] + 1, vocab), dim=1).values[:, -1:]
    at = torch.nonzero((scores >= least) & (scores > -math.inf))
    r, t = at[:, 0], at[:, 1]
    value = scores[r, t]
    order = torch.argsort(value, descending=True, stable=True)
    order = order[torch.argsort(session[r[order]], stable=True)]
    r, t, value = r[order], t[order], value[order]
    s = session[r]
    begin = torch.searchsorted(s, torch.arange(width.numel(), device=DEVICE))
    ends = t == st["end"]
    place = torch.arange(s.numel(), device=DEVICE) - begin[s]              # among all of the session's
    before = torch.cumsum((~ends).long(), 0) - (~ends).long()             # among those that go on
    going = before - torch.cat([before, before.new_zeros(1)])[begin[s]]
    to = torch.where(~ends & (going < width[s]), cu_next[s] + going, cu_next[-1])
    total = st["parents"].numel()
    put = lambda fill, v, dt: torch.full((total + 1,), fill, dtype=dt, device=DEVICE).scatter(0, to, v.to(dt))[:total]  # noqa: E731
    ended = torch.full((rows + 1,), -math.inf, dtype=torch.float64, device=DEVICE).scatter(
        0, torch.where(ends & (place < width[s]), r, rows), value)[:rows]
    return {"parents": put(-1, r, torch.int32), "tokens": put(-1, t, torch.int32), "scores": put(-math.inf, value, torch.float64).float(),
            "end_scores": ended.float()}


def _blocks(st):
    """(blocks of whole tokens, blocks in use, blocks held) of every row."""
    lens, bs = st["lens"].long(), st["bs"]
    used = (lens + bs - 1) // bs
    return lens // bs, used, torch.maximum(used, st["held"].long())


def _plus(refs, ids, amount):
    """refs with `amount` added at `ids`; ids outside the pool count for nothing."""
    n = refs.numel()
    inside = (ids >= 0) & (ids < n)
    more = torch.cat([refs, refs.new_zeros(1)])
    return more.index_add(0, torch.where(inside, ids, n).reshape(-1).long(), amount.to(refs.dtype).reshape(-1))[:n]


def _plain_fork(st):
    rows, out, bs, free = st["lens"].numel(), st["parents"].numel(), st["bs"], st["free"]
    whole, used, held = _blocks(st)
    lens, table, n = st["lens"].long(), st["table"], st["refs"].numel()
    i = torch.arange(out, device=DEVICE)
    valid = (st["parents"] >= 0) & (st["parents"] < rows)
    p = st["parents"].long().clamp(0, rows - 1)
    first = torch.full((rows + 1,), out, device=DEVICE).scatter_reduce(0, torch.where(valid, p, rows), i, "amin")
    keeps = valid & (first[p] == i)                                # a row's first child goes on in its last block
    copies = valid & ~keeps & (whole[p] < used[p])                 # the others get copies of what is filled of it
    place = torch.cumsum(copies.long(), 0) - copies.long() + st["begin"].long()
    new = torch.where(copies & (place < free.numel()), free[place.clamp(max=free.numel() - 1)], torch.full_like(free[:1], -1))
    cols = torch.arange(table.shape[1], device=DEVICE)
    held_out = torch.where(valid, torch.where(keeps, held[p], used[p]), torch.zeros_like(p))
    entry = torch.where(copies[:, None] & (cols == whole[p][:, None]), new[:, None], table[p])
    table_out = torch.where(cols < held_out[:, None], entry, st["table_out"])
    children = torch.zeros(rows + 1, dtype=torch.int64, device=DEVICE).index_add(0, torch.where(valid, p, rows), torch.ones_like(p))[:rows]
    change = torch.where(cols < whole[:, None], children[:, None] - 1,
                         torch.where(cols < held[:, None], -(children == 0).long()[:, None], torch.zeros_like(cols)))
    refs = _plus(_plus(st["refs"], table, change), new, torch.ones_like(new))
    made = new >= 0
    from_ = torch.where(made, table[p, whole[p].clamp(max=table.shape[1] - 1)], torch.full_like(new, -1))
    return {"table": table_out, "lens": torch.where(valid, lens[p], torch.zeros_like(p)).int(), "held": held_out.int(), "refs": refs,
            "copy_src": from_, "copy_dst": new, "copy_tokens": torch.where(made, lens[p] % bs, torch.zeros_like(p)).int(),
            "taken": (st["begin"] + copies.sum()).int()}


def _plain_copy(st):
    src, dst, (_, _, bs, _, _) = st["src"].long(), st["dst"].long(), st["k_pool"].shape
    filled = torch.full_like(src, bs) if st["tokens"] is None else st["tokens"].long()
    place = torch.arange(bs, device=DEVICE)
    pair, slot = torch.nonzero((src >= 0)[:, None] & (place < filled[:, None]), as_tuple=True)
    for pool in (st["k_pool"], st["v_pool"]):
        rows = pool.view(pool.shape[0], -1, *pool.shape[3:])
        rows[:, dst[pair] * bs + slot] = rows[:, src[pair] * bs + slot]
    return _pools(st)


def _plain_free(st):
    table, drop = st["table"], st["drop"] != 0
    cols = torch.arange(table.shape[1], device=DEVICE)
    gone = drop[:, None] & (cols < _blocks(st)[2][:, None])
    refs = _plus(st["refs"], table, -gone.long())
    n = refs.numel()
    unused = refs <= 0
    place = torch.cumsum(unused.long(), 0) - 1
    listed_ = torch.full((n + 1,), -1, dtype=torch.int32, device=DEVICE).scatter(
        0, torch.where(unused, place, n), torch.arange(n, dtype=torch.int32, device=DEVICE))[:n]
    nothing = torch.zeros_like(st["lens"])
    return {"refs": refs, "free": listed_, "n_free": unused.sum().int().view(1), "lens": torch.where(drop, nothing, st["lens"]),
            "held": torch.where(drop, nothing, _blocks(st)[2].int())}


def _plain_compact(st):
    refs, table, n, moves = st["refs"], st["table"], st["refs"].numel(), st["copy_src"].numel()
    b = torch.arange(n, device=DEVICE)
    used = refs > 0
    n_used = used.sum()
    keep = n_used if st["n_keep"] < 0 else torch.full_like(n_used, st["n_keep"])
    leaves, takes = used & (b >= keep), ~used & (b < keep)
    k_from, k_to = torch.cumsum(leaves.long(), 0) - 1, torch.cumsum(takes.long(), 0) - 1
    moved = torch.minimum(leaves.sum(), takes.sum()).clamp(max=moves)
    put = lambda mask, k: torch.full((moves + 1,), -1, dtype=torch.int32, device=DEVICE).scatter(  # noqa: E731
        0, torch.where(mask & (k < moved), k, moves), b.int())[:moves]
    src, dst = put(leaves, k_from), put(takes, k_to)
    far = torch.cat([dst, dst.new_full((1,), -1)])
    moves_away = leaves & (k_from < moved)
    block_map = torch.where(moves_away, far[k_from.clamp(0, moves)], b.int())
    back = torch.cat([src, src.new_zeros(1)])
    taken = takes & (k_to < moved)
    refs_after = torch.where(moves_away, torch.zeros_like(refs),
                             torch.where(taken, refs[back[k_to.clamp(0, moves)].clamp(min=0).long()], refs))
    cols = torch.arange(table.shape[1], device=DEVICE)
    inside = (cols < _blocks(st)[2][:, None]) & (table >= 0) & (table < n)
    return {"table": torch.where(inside, block_map[table.clamp(0, n - 1).long()], table), "refs": refs_after, "map": block_map,
            "copy_src": src, "copy_dst": dst, "counts": torch.stack([n_used, moved, leaves.sum() - moved]).int()}


def _pools(st):
    whole = torch.int16 if st["k_pool"].element_size() == 2 else torch.int32
    return {"k_pool": st["k_pool"].view(whole), "v_pool": st["v_pool"].view(whole)}


_PLAIN = {"beam": _plain_beam, "fork": _plain_fork, "copy": _plain_copy, "free": _plain_free, "compact": _plain_compact}


# ------------------------------------------------------------------------------------------------------------------
# the package's calls
# ------------------------------------------------------------------------------------------------------------------
def _workspace(st, size):
    """What a server holds on to: made by a state's first call."""
    if "workspace" not in st:
        n = size()
        st["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEVICE) if n else None
    return st["workspace"]


def _own(st):
    import paper_2412_16434_amd as S
    op = st["op"]
    if op == "beam":
        space = _workspace(st, lambda: S.beam_select_workspace_bytes(*st["logits"].shape, st["max_next"]))
        S.beam_select(st["logits"], st["scores"], st["cu"], st["cu_next"], st["max_next"], st["parents"], st["tokens"],
                      st["next_scores"], end_token=st["end"], end_scores=st["end_scores"], workspace=space)
        return {"parents": st["parents"], "tokens": st["tokens"], "scores": st["next_scores"], "end_scores": st["end_scores"]}
    if op == "fork":
        S.kv_fork(st["parents"], st["lens"], st["table"], st["refs"], st["free"], st["bs"], st["table_out"], st["lens_out"],
                  st["refs_after"], st["copy_src"], st["copy_dst"], st["copy_tokens"], held_blocks=st["held"],
                  held_out=st["held_out"], free_begin=st["begin"], blocks_taken=st["taken"])
        return {"table": st["table_out"], "lens": st["lens_out"], "held": st["held_out"], "refs": st["refs_after"],
                "copy_src": st["copy_src"], "copy_dst": st["copy_dst"], "copy_tokens": st["copy_tokens"], "taken": st["taken"]}
    if op == "copy":
        if "cache" not in st:
            st["cache"] = S.KVCache(st["k_pool"], st["v_pool"])
        S.kv_copy_blocks(st["cache"], st["src"], st["dst"], st["tokens"])
        return _pools(st)
    if op == "free":
        space = _workspace(st, lambda: S.kv_free_workspace_bytes(st["refs"].numel()))
        S.kv_free(st["drop"], st["lens"], st["table"], st["refs"], st["bs"], st["refs_after"], st["free"], st["n_free"],
                  held_blocks=st["held"], lens_after=st["lens_after"], held_after=st["held_after"], workspace=space)
        return {"refs": st["refs_after"], "free": st["free"], "n_free": st["n_free"], "lens": st["lens_after"], "held": st["held_after"]}
    space = _workspace(st, lambda: S.kv_compact_workspace_bytes(st["refs"].numel()))
    S.kv_compact(st["refs"], st["n_keep"], st["lens"], st["table"], st["bs"], st["table_out"], st["refs_after"], st["map"],
                 st["copy_src"], st["copy_dst"], st["counts"], held_blocks=st["held"], workspace=space)
    return {"table": st["table_out"], "refs": st["refs_after"], "map": st["map"], "copy_src": st["copy_src"],
            "copy_dst": st["copy_dst"], "counts": st["counts"]}


def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


def exact(case, seed):
    """The scores in 64 bits, session by session; all other outputs are whole numbers."""
    if case["op"] != "beam":
        return None
    st, (beams, wide), out, at, ended = _prepare_beam(case, seed), _widths(case), [], 0, []
    for b, w in zip(beams, wide):
        x = torch.log_softmax(st["logits"][at:at + b].double(), dim=1) + st["scores"][at:at + b, None].double()
        x = torch.nan_to_num(x, nan=-math.inf, neginf=-math.inf)
        if st["end"] >= 0:
            e = x[:, st["end"]].clone()
            # among the best of all: at least as good as the last of them
            last = torch.topk(x.flatten(), min(w, x.numel())).values[-1] if w <= x.numel() else -math.inf
            ended.append(torch.where(e >= last, e, torch.full_like(e, -math.inf)))
            x[:, st["end"]] = -math.inf
        else:
            ended.append(torch.full((b,), -math.inf, dtype=torch.float64, device=DEVICE))
        best = torch.topk(x.flatten(), min(w, x.numel())).values
        out.append(torch.nn.functional.pad(best, (0, w - best.numel()), value=-math.inf))
        at += b
    return {"parents": None, "tokens": None, "scores": torch.cat(out), "end_scores": torch.cat(ended)}


# ------------------------------------------------------------------------------------------------------------------
# drawn cases
# ------------------------------------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _drawn(op, rng):
    case = dict(op=op, lens=rng.randrange(1 << 30))
    if op == "beam":
        case.update(dtype=rng.choice(["bf16", "fp32"]), sessions=_log(rng, 1, 256), vocab=_log(rng, 300, 160000),
                    masked=rng.choice([0, 0, 50, 99]), end=rng.choice([0, 1, 1]), b_hi=_log(rng, 1, 32))
        case["b_lo"], case["w_hi"] = rng.choice([case["b_hi"], max(1, case["b_hi"] // 4), 1]), min(64, 2 * case["b_hi"])
        return case
    case["bs"] = rng.choice([16, 16, 16, 32, 64, 8, 24, 1])
    if op == "copy":
        case.update(dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]), layers=rng.choice([1, 16, 28, 32]),
                    hkv=rng.choice([1, 2, 4, 8, 8, 8]), d=rng.choice([128, 128, 64]), pairs=_log(rng, 1, 1024), whole=rng.choice([0, 1]),
                    skip=rng.choice([0, 45, 90]))
        return case
    case.update(sessions=_log(rng, 1, 256), beams=_log(rng, 1, 32), p_hi=_log(rng, 1, 16384), g_hi=_log(rng, 1, 1000),
                blocks=_log(rng, 64, 131072))
    case["p_lo"] = case["p_hi"] // rng.choice([1, 2, 8, 100000])
    if op == "fork":
        case.update(out=rng.choice([case["beams"], _log(rng, 1, 32)]), short=rng.choice([0, 0, 0, 2]))
    elif op == "free":
        case.update(drop=rng.choice([0, 10, 50, 100]))
    else:
        case.update(keep=rng.choice([0, 0, 50, 75]))
    return case


def draw(rng):
    """One more case of the listed ones' ranges: an operator, then its sizes (spread over their logarithm)."""
    op = rng.choice(["beam", "beam", "fork", "copy", "free", "compact"])
    for _ in range(1000):
        case = _drawn(op, rng)
        w = work(case)
        if op == "beam":
            # (the plain form holds some copies of the logits in 64 bits)
            ok = w["bytes"] <= 1.3e8 and w["flops"] <= 2.6e8
        elif op == "copy":
            ok = w["bytes"] <= 1.8e9 and case["pairs"] * case["bs"] * case["layers"] * case["hkv"] * case["d"] * _elem(case) <= 1e9
        else:
            rows = case["sessions"] * max(case["beams"], case.get("out", 1))
            ok = w["bytes"] <= 3e6 and rows <= 2048 and rows * int(_own_blocks(case)[0].max()) <= 600000
        if ok:
            return case
    raise RuntimeError("no case in range")
