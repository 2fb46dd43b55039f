"""The speculative step's operators at the sizes where a kernel's way of working changes: calls of a million tokens, rows of every
number of 16-byte pieces, trees around the edges of chunks and stages."""
import numpy as np
import pytest
import torch

import draft_ref as R
import paper_2412_16434_amd as S
from gpu_util import DEV
from test_gpu_draft_step import Draft, check_mask, check_tables, cumulated, dev, random_parents

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prefix,new,bs,total", [
    ([5, 0, 77, 3, 0], [700001, 3, 0, 400000, 1], 16, None),
    ([0, 15, 16], [1048575, 0, 1], 16, None),                    # exactly 2^20
    ([0, 9], [1048570, 5], 7, None),                             # one less
    ([31] * 1100, [957] * 1100, 24, None),                       # more sessions than are added up at a time
    ([3, 4], [500000, 30], 64, 1 << 20),                         # more tokens announced than the sessions have
    ([3, 4], [900000, 900000], 1, (1 << 20) + 5)])               # and fewer
def test_tables_of_a_million_tokens(prefix, new, bs, total):
    check_tables(prefix, new, bs, 21, total=total)


@pytest.mark.parametrize("total", [511, 512, 513, 1023, 1025])
def test_tables_around_a_workgroups_tokens(total):
    check_tables([4, 0, 30], [total - 7, 0, 7], 16, 22)
    check_tables([4], [total], 16, 23)
    check_tables(np.zeros(1024, int), [0] * 1023 + [total], 16, 24)       # all tokens in the last session of a chunk
    check_tables(np.zeros(1025, int), [0] * 1024 + [total], 16, 25)       # and in the first of the next
    check_tables(np.zeros(600, int), [1, 0] * 300, 16, 26)


def test_slot_maps_and_positions_at_odd_addresses():
    n, bs = 700, 16
    table = torch.full((1, 50), -1, dtype=torch.int32, device=DEV)
    slots = torch.full((n + 1,), 77, dtype=torch.int64, device=DEV)
    positions = torch.full((n + 1,), 77, dtype=torch.int32, device=DEV)
    S.build_tables(dev([3], np.int32), dev([n], np.int32), table, torch.arange(50, dtype=torch.int32, device=DEV), bs, 60, n,
                   slot_map=slots[1:], positions=positions[1:], held_blocks=dev([0], np.int32))
    torch.cuda.synchronize()
    want = R.build_tables([3], [n], np.full((1, 50), -1, np.int32), np.arange(50), bs, 60, n)
    assert int(slots[0]) == 77 and int(positions[0]) == 77
    assert np.array_equal(slots[1:].cpu().numpy(), want["slots"]) and np.array_equal(positions[1:].cpu().numpy(), want["positions"])


@pytest.mark.parametrize("n", [3, 255, 256, 449, 513])
@pytest.mark.parametrize("words", [9, 16, 17, 64])
def test_masks_of_rows_wider_than_a_stage(n, words):
    rng = np.random.default_rng(n + words)
    check_mask([random_parents(n, rng, 7), random_parents(5, rng, 2), random_parents(n // 2, rng, 400)], words=words, prefix=[1, 2, 3])


def test_chains_and_stars_of_the_largest_size():
    check_mask([np.arange(-1, 4095, dtype=np.int32)])
    check_mask([np.concatenate([[-1], np.zeros(4095)]).astype(np.int32)])


@pytest.mark.parametrize("sizes", [[129], [64, 64], [65, 200]])
def test_accepted_paths_through_several_chunks(sizes):
    """Chains that agree everywhere, and ones whose every node hangs on one of an earlier chunk."""
    rng = np.random.default_rng(sum(sizes))
    for parents in ([np.arange(-1, k - 1).astype(np.int32) for k in sizes],
                    [np.maximum(np.arange(k) - 64, np.where(np.arange(k) > 0, 0, -1)).astype(np.int32) for k in sizes]):
        draft = [rng.integers(0, 50, k).astype(np.int32) for k in sizes]
        target = []
        for d, p in zip(draft, parents):            # every node's first child agrees with it
            t = np.full(len(d), 99, np.int32)
            for i in range(len(d) - 1, 0, -1):
                t[p[i]] = d[i]
            target.append(t)
        cu = cumulated(sizes)
        rows, count, nxt = (torch.full((k,), 77, dtype=torch.int32, device=DEV) for k in (int(cu[-1]), len(sizes), len(sizes)))
        S.tree_accept(dev(np.concatenate(draft)), dev(np.concatenate(parents)), dev(np.concatenate(target)), dev(cu), None, rows,
                      count, nxt)
        torch.cuda.synchronize()
        for s, (d, p, t) in enumerate(zip(draft, parents, target)):
            path = R.accept(d, p, t)
            want = [cu[s] + i for i in path] + [-1] * (len(d) - len(path))
            assert rows[cu[s]:cu[s + 1]].tolist() == want and int(count[s]) == len(path) and int(nxt[s]) == t[path[-1]]


@pytest.mark.parametrize("hkv,d", [(1, 8), (5, 100), (8, 64), (9, 64), (3, 344), (24, 128), (33, 64)])
@pytest.mark.parametrize("accepted", [1, 2, 15, 64, 130])
def test_commit_of_rows_of_every_width(hkv, d, accepted):
    rng = np.random.default_rng(hkv * accepted)
    layers, bs, n_blocks, n_rows, n_entries = 2, 4, 50, 150, 200
    pools = [torch.randn((layers, n_blocks, bs, hkv, d), device=DEV).bfloat16() for _ in range(2)]
    new = [torch.randn((layers, n_rows, hkv, d), device=DEV).bfloat16() for _ in range(2)]
    rows, slots = np.full(n_entries, -1, np.int32), rng.permutation(n_blocks * bs)[:n_entries].astype(np.int64)
    for t in rng.permutation(n_entries)[:accepted]:
        rows[t] = rng.integers(0, n_rows)
    want = [p.clone().view(layers, n_blocks * bs, hkv, d) for p in pools]
    for t in np.flatnonzero(rows >= 0):
        for w, x in zip(want, new):
            w[:, int(slots[t])] = x[:, int(rows[t])]
    S.kv_commit(S.KVCache(*pools), *new, dev(rows), dev(slots))
    torch.cuda.synchronize()
    for p, w in zip(pools, want):
        assert torch.equal(p.view_as(w), w)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bs", [2, 4, 8, 12, 20, 24, 40, 56, 1000])
@pytest.mark.parametrize("prefix,new", [([0, 3, 700], [33, 20, 64]), ([1990], [40]), ([65, 1000], [3, 8])])
def test_attention_over_blocks_of_every_size(d, bs, prefix, new):
    Draft(prefix, new, "bf16", d, bs=bs, hkv=2, g=4, seed=31).check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bs", [8, 24])
def test_block_ids_outside_the_cache_under_wide_tiles(d, bs):
    draft = Draft([300, 45], [40, 36], "bf16", d, bs=bs, seed=32)
    draft.table[0, 2], draft.table[0, 7], draft.table[1, 0] = -5, 1 << 30, draft.k_pool.shape[0]
    draft.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bs", [2, 8, 12, 16, 24, 40])
@pytest.mark.parametrize("prefix,new", [([0, 3, 700], [33, 20, 64]), ([1990], [40]), ([65, 8, 128, 136], [3, 16, 1, 17])])
def test_fp32_attention_over_blocks_of_every_size(d, bs, prefix, new):
    Draft(prefix, new, "fp32", d, bs=bs, hkv=2, g=3, tree="bits", seed=33).check()


@pytest.mark.parametrize("bs", [8, 24, 16])
def test_fp32_block_ids_outside_the_cache(bs):
    draft = Draft([300, 45], [6, 6], "fp32", 128, bs=bs, seed=34)
    draft.table[0, 2], draft.table[0, 7], draft.table[1, 0] = -5, 1 << 30, draft.k_pool.shape[0]
    draft.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("bs", [16, 8])
@pytest.mark.parametrize("hkv,g,new_hi", [(4, 1, 5), (2, 4, 16), (1, 7, 9)])
def test_many_sessions_with_hardly_a_cache(dtype, d, bs, hkv, g, new_hi):
    rng = np.random.default_rng(bs + hkv)
    prefix, new = rng.integers(0, 40, 140), rng.integers(0, new_hi + 1, 140)
    prefix[7], new[7] = 200, new_hi
    draft = Draft(prefix, new, dtype, d, bs=bs, hkv=hkv, g=g, tree="bits", seed=35)
    draft.check()
    draft.check(max_prefix=1)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("tree", ["tree", "bits", "none"])
def test_wide_trees_whose_tiles_see_only_their_beginning(dtype, d, tree):
    """Tiles of rows far apart in a large tree; rows that see nothing of it, with and without a cache."""
    Draft([0, 70], [200, 131], dtype, d, hkv=1, g=4, tree=tree, seed=36).check()
    Draft([0], [256], dtype, d, hkv=2, g=1, tree=tree, seed=37).check()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
def test_many_tiles_are_not_cut(dtype, d):
    rng = np.random.default_rng(38)
    prefix, new = rng.integers(0, 500, 70), rng.integers(20, 34, 70)
    prefix[3], new[5] = 0, 0
    Draft(prefix, new, dtype, d, hkv=4, g=4, tree="bits", seed=38).check()
