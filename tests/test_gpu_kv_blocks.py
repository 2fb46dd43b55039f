"""symph_kv_fork, symph_kv_free, symph_kv_compact and symph_kv_copy_blocks against loops over their definitions."""
import numpy as np
import pytest
import torch

import beam_ref as R
import paper_2412_16434_amd as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LEFT = 77


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).to(DEV).contiguous()


def _left(*shape):
    return torch.full(shape, LEFT, dtype=torch.int32, device=DEV)


def _same(got, want):
    torch.cuda.synchronize()
    for name, value in want.items():
        if got.get(name) is not None:
            have = got[name].cpu().numpy()
            assert np.array_equal(have, np.asarray(value, np.int32).reshape(have.shape)), (name, have, value)


def _fork(parents, lens, held, table, refs, free, bs, begin=0, with_held=True, with_begin=True):
    n_out = len(parents)
    got = dict(table_out=_left(n_out, table.shape[1]), lens_out=_left(n_out), refs_after=_left(len(refs)), copy_src=_left(n_out),
               copy_dst=_left(n_out), copy_tokens=_left(n_out), held_out=_left(n_out) if with_held else None, blocks_taken=_left(1))
    out = np.full((n_out, table.shape[1]), LEFT, np.int32)
    inputs = [_i32(x) for x in (parents, lens, table, refs, free)]
    before = [x.clone() for x in inputs]
    S.kv_fork(*inputs, bs, held_blocks=_i32(held) if with_held else None, free_begin=_i32([begin]) if with_begin else None, **got)
    _same(got, R.fork(np.asarray(parents), lens, held if with_held else np.zeros_like(held), table, refs, free, begin, bs, out))
    assert all(torch.equal(a, b) for a, b in zip(inputs, before))
    return got


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("bs", [1, 5, 16, 64])
@pytest.mark.parametrize("sessions,beams,longest", [(1, 1, 1), (1, 4, 100), (7, 3, 333), (40, 8, 60), (2, 5, 5000)])
def test_forks(sessions, beams, longest, bs, wide):
    rs = np.random.RandomState(sessions + bs)
    lens, held, table, refs, free = R.shared_pages(rs, sessions, beams, bs, longest, 4 * sessions * beams * (longest // bs + 4))
    rows = sessions * beams
    if wide:  # (tables of many entries take two launches)
        table = np.pad(table, ((0, 0), (0, 16400 // rows)), constant_values=-1)
    for n_out in (rows, 1, 3 * rows + 1):
        parents = rs.randint(0, rows, size=n_out) if n_out != rows else np.arange(rows) // beams * beams + rs.randint(0, beams, size=rows)
        parents = np.where(rs.random_sample(n_out) < 0.1, -1, parents)
        got = _fork(parents, lens, held, table, refs, free, bs, begin=int(rs.randint(0, 2)))
        # what nobody holds, and only that, has no count: the invariant that the next step builds on
        n_free = int((got["refs_after"].cpu().numpy() == 0).sum())
        held_out, table_out = got["held_out"].cpu().numpy(), got["table_out"].cpu().numpy()
        held_by = np.concatenate([table_out[j, :held_out[j]] for j in range(n_out)] + [np.empty(0, int)])
        assert n_free == len(refs) - len(np.unique(held_by[held_by >= 0]))


def test_a_prompt_becomes_beams():
    table = np.array([[4, 2, 9, -1]], np.int32)
    refs = np.bincount([4, 2, 9], minlength=12).astype(np.int32)
    got = _fork([0, 0, 0], np.array([37]), np.array([0]), table, refs, np.array([7, 1, 3]), 16)
    assert got["table_out"].tolist() == [[4, 2, 9, LEFT], [4, 2, 7, LEFT], [4, 2, 1, LEFT]]
    assert got["copy_tokens"].tolist() == [0, 5, 5] and got["refs_after"].tolist() == [0, 1, 3, 0, 3, 0, 0, 1, 0, 1, 0, 0]


@pytest.mark.parametrize("wide", [False, True])
def test_lists_that_end_too_early_and_blocks_outside(wide):
    rs = np.random.RandomState(3)
    lens, held, table, refs, free = R.shared_pages(rs, 4, 4, 16, 200, 600)
    if wide:
        table = np.pad(table, ((0, 0), (0, 1100)), constant_values=-1)
    parents = np.repeat(np.arange(16), 2)
    lens[:] = np.maximum(lens, 1) | 1  # (no full last block)
    for bad, begin in ((free[:5], 0), (free[:5], 4), (free, 10_000), (free, -3), (free[:0], 0), (np.array([-1, 600, 5]), 0)):
        _fork(parents, lens, held, table, refs, bad, 16, begin)
    odd = table.copy()
    odd[2], odd[5, 0], odd[7, ::2] = -1, 600, 10 ** 9
    _fork(parents, lens, held, odd, refs, free, 16)
    _fork([-1, -2 ** 31, 16, 2 ** 31 - 1, 15], lens, held, table, refs, free, 16)
    _fork(parents, lens * 1000, held * 1000, table, refs, free, 16)        # longer than their table rows
    _fork(parents, np.where(lens % 3 == 0, -lens, lens), held, table, refs, free, 16)
    _fork(parents, lens, held, table, refs, free, 16, with_held=False, with_begin=False)
    _fork(parents, np.full(16, 2 ** 31 - 1), np.full(16, 2 ** 31 - 1), table, refs, free, 2 ** 31 - 1)


def test_empty_tables():
    none = np.zeros(0, np.int32)
    refs = np.array([0, 2, 1], np.int32)
    _fork(none, np.array([20]), np.array([0]), np.array([[1, 2]], np.int32), refs, np.array([0]), 16, begin=7)   # every row goes
    _fork([0, 0], none, none, np.zeros((0, 3), np.int32), refs, np.array([0]), 16)
    _fork(none, none, none, np.zeros((0, 3), np.int32), refs, none, 16)
    _fork([0, 0], np.array([0]), np.array([0]), np.zeros((1, 0), np.int32), refs, none, 16)


def test_many_rows():
    rs = np.random.RandomState(8)
    lens, held, table, refs, free = R.shared_pages(rs, 512, 16, 16, 40, 100_000)
    parents = np.arange(8192) // 16 * 16 + rs.randint(0, 16, size=8192)
    got = dict(table_out=_left(*table.shape), lens_out=_left(8192), refs_after=_left(len(refs)), copy_src=_left(8192),
               copy_dst=_left(8192), copy_tokens=_left(8192), held_out=_left(8192), blocks_taken=_left(1))
    S.kv_fork(*(_i32(x) for x in (parents, lens, table, refs, free)), 16, held_blocks=_i32(held), **got)
    first = np.full(8192, 8192)
    np.minimum.at(first, parents, np.arange(8192))
    copies = (first[parents] != np.arange(8192)) & (lens[parents] % 16 > 0)
    want = np.full(8192, -1)
    want[copies] = free[:copies.sum()]
    _same(got, dict(copy_dst=want, lens_out=lens[parents], blocks_taken=[copies.sum()]))
    held_out, table_out = got["held_out"].cpu().numpy(), got["table_out"].cpu().numpy()
    counts = np.bincount(np.concatenate([table_out[j, :held_out[j]] for j in range(8192)]), minlength=len(refs))
    _same(got, dict(refs_after=counts))


def _free(drop, lens, held, table, refs, bs, with_held=True, taken=None, begin=0, end=0):
    n, n_blocks = len(drop), len(refs)
    more = {} if taken is None else dict(taken_blocks=_i32(taken), taken_begin=_i32([begin]), taken_end=_i32([end]))
    got = dict(refs_after=_left(n_blocks), free_blocks=_left(n_blocks), n_free=_left(1), lens_after=_left(n), held_after=_left(n))
    space = torch.full((S.kv_free_workspace_bytes(n_blocks),), 255, dtype=torch.uint8, device=DEV)
    S.kv_free(_i32(drop), _i32(lens), _i32(table), _i32(refs), bs, held_blocks=_i32(held) if with_held else None, workspace=space, **got,
              **more)
    _same(got, R.free(drop, lens, held if with_held else np.zeros_like(held), table, refs, bs, [] if taken is None else taken, begin, end))
    return got


@pytest.mark.parametrize("bs", [1, 5, 16])
@pytest.mark.parametrize("n_blocks", [1, 2, 255, 1023, 1025, 5000, 70001])
def test_frees(n_blocks, bs):
    rs = np.random.RandomState(n_blocks)
    longest = max(0, min(300, n_blocks * bs // 40 - 4 * bs))
    beams, sessions = (4, 3) if n_blocks > 200 else (1, 1)
    lens, held, table, refs, _ = R.shared_pages(rs, sessions, beams, bs, longest, n_blocks, ahead=1 if n_blocks > 200 else 0)
    for drop in (np.zeros(len(lens), int), np.ones(len(lens), int), rs.randint(-1, 2, size=len(lens))):
        _free(drop, lens, held, table, refs, bs)
    _free(drop, lens, held, table, refs, bs, with_held=False)
    _free(drop, lens, held, np.pad(table, ((0, 0), (0, 16400)), constant_values=0), refs, bs)   # (not the small call's kernel)
    _free(drop, lens, held, table, rs.randint(-2, 3, size=n_blocks), bs)   # counts that do not belong to the table


@pytest.mark.parametrize("n_blocks", [900, 20000])
def test_blocks_that_were_taken_since(n_blocks):
    """A list of which some entries were taken: parts of it, none, more than there are, ids outside the pool, blocks of dropped rows."""
    rs = np.random.RandomState(4)
    lens, held, table, refs, free = R.shared_pages(rs, 4, 3, 16, 200, n_blocks)
    drop = rs.randint(0, 2, size=12)
    for taken, begin, end in ((free, 0, 30), (free, 7, 8), (free, 9, 9), (free, 50, 20), (free[:20], -5, 10 ** 9), (free[:0], 0, 3),
                              (free, 2 ** 31 - 1, 2 ** 31 - 1), (np.array([-1, n_blocks, free[0], 10 ** 9]), 0, 4)):
        _free(drop, lens, held, table, refs, 16, taken=taken, begin=begin, end=end)
    row = int(np.flatnonzero((drop != 0) & (held > 0))[0])
    fresh = refs.copy()
    fresh[table[row, held[row] - 1]] -= 1      # (a block that a dropped row holds, and that is not counted yet)
    _free(drop, lens, held, table, fresh, 16, taken=table[row, held[row] - 1:held[row]], begin=0, end=1)
    ids, count, after = _left(n_blocks), _left(1), _left(n_blocks)
    space = torch.empty(S.kv_free_workspace_bytes(n_blocks), dtype=torch.uint8, device=DEV)
    S.kv_free(None, None, None, _i32(refs), 16, after, ids, count, workspace=space, taken_blocks=_i32(free), taken_end=_i32([5]))
    want = R.free([], [], [], np.zeros((0, 1), int), refs, 16, free, 0, 5)
    _same(dict(refs_after=after, free_blocks=ids, n_free=count), {k: want[k] for k in ("refs_after", "free_blocks", "n_free")})


def test_a_list_without_rows_and_a_large_pool():
    for n_blocks in (1, 3_000_001):     # (more tiles than workgroups)
        refs = (torch.rand(n_blocks, generator=torch.Generator().manual_seed(1)) < 0.5).int()
        after, ids, count = _left(n_blocks), _left(n_blocks), _left(1)
        space = torch.empty(S.kv_free_workspace_bytes(n_blocks), dtype=torch.uint8, device=DEV)
        S.kv_free(None, None, None, refs.to(DEV), 16, after, ids, count, workspace=space)
        want = torch.nonzero(refs <= 0)[:, 0].int()
        n = want.numel()
        assert count.item() == n and torch.equal(ids[:n].cpu(), want) and bool((ids[n:] == -1).all()) and torch.equal(after.cpu(), refs)


def test_lengths_in_place():
    rs = np.random.RandomState(5)
    lens, held, table, refs, _ = R.shared_pages(rs, 30, 4, 16, 3000, 40000)
    drop = rs.randint(0, 2, size=120)
    want = R.free(drop, lens, held, table, refs, 16)
    l, h, n = _i32(lens), _i32(held), len(refs)
    after, ids, count = _left(n), _left(n), _left(1)
    space = torch.empty(S.kv_free_workspace_bytes(n), dtype=torch.uint8, device=DEV)
    S.kv_free(_i32(drop), l, _i32(table), _i32(refs), 16, after, ids, count, held_blocks=h, lens_after=l, held_after=h, workspace=space)
    _same(dict(lens_after=l, held_after=h, refs_after=after, free_blocks=ids, n_free=count), want)


def _compact(refs, n_keep, lens, held, table, bs, n_pairs, in_place=False):
    n, t = len(refs), _i32(table)
    got = dict(table_out=t if in_place else _left(*table.shape), refs_after=_left(n), block_map=_left(n), copy_src=_left(n_pairs),
               copy_dst=_left(n_pairs), counts=_left(3))
    space = torch.full((S.kv_compact_workspace_bytes(n),), 255, dtype=torch.uint8, device=DEV)
    S.kv_compact(_i32(refs), n_keep, _i32(lens), t, bs, held_blocks=_i32(held), workspace=space, **got)
    want = R.compact(refs, n_keep, lens, held, table, bs, n_pairs, table if in_place else np.full_like(table, LEFT))
    _same(got, want)
    return got


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n_blocks", [1, 2, 300, 1024, 2049, 9000])
def test_compactions(n_blocks, in_place):
    rs = np.random.RandomState(n_blocks)
    beams, sessions = (3, 4) if n_blocks > 200 else (1, 1)
    longest = max(0, min(900, n_blocks // 3 - 20))
    lens, held, table, refs, _ = R.shared_pages(rs, sessions, beams, 16, longest, n_blocks, ahead=1 if n_blocks > 200 else 0)
    for n_keep in (-1, 0, 1, n_blocks // 2, n_blocks - 1, n_blocks, 2 ** 31 - 1, -(2 ** 31), 1024):
        for n_pairs in (n_blocks, 5, 0):
            _compact(refs, n_keep, lens, held, table, 16, n_pairs, in_place)
    _compact(refs, -1, lens, held, np.pad(table, ((0, 0), (0, 16400)), constant_values=0), 16, n_blocks, in_place)


def test_compactions_of_full_empty_and_large_pools():
    none = np.zeros(0, np.int32)
    for refs in (np.zeros(3000, np.int32), np.ones(3000, np.int32), np.arange(3000, dtype=np.int32) % 2, np.full(3000, -1, np.int32)):
        for n_keep in (-1, 700, 1500):
            _compact(refs, n_keep, none, none, np.zeros((0, 4), np.int32), 16, 1500)
    n = 3_000_001                           # (more tiles than workgroups)
    refs = (torch.rand(n, generator=torch.Generator().manual_seed(2)) < 0.3).int().to(DEV)
    src, dst, counts, after, where = _left(n), _left(n), _left(3), _left(n), _left(n)
    space = torch.empty(S.kv_compact_workspace_bytes(n), dtype=torch.uint8, device=DEV)
    empty = torch.zeros(0, dtype=torch.int32, device=DEV)
    S.kv_compact(refs, -1, empty, torch.zeros((0, 1), dtype=torch.int32, device=DEV), 16, torch.zeros((0, 1), dtype=torch.int32, device=DEV),
                 after, where, src, dst, counts, workspace=space)
    used = int((refs > 0).sum())
    a, b = torch.nonzero(refs[used:] > 0)[:, 0] + used, torch.nonzero(refs[:used] <= 0)[:, 0]
    m = a.numel()
    assert counts.tolist() == [used, m, 0] and torch.equal(src[:m].long(), a) and torch.equal(dst[:m].long(), b)
    assert bool((src[m:] == -1).all()) and bool((dst[m:] == -1).all()) and torch.equal(where[a].long(), b)
    assert bool((after[:used] > 0).all()) and bool((after[used:] == 0).all())


def _pools(layers, n_blocks, bs, hkv, d, dtype, seed, pad=0):
    """Pools of random bits, `pad` elements between blocks; (cache, the two pools as whole numbers)."""
    width = {torch.bfloat16: torch.int16, torch.float32: torch.int32}[dtype]
    g = torch.Generator().manual_seed(seed)
    block = bs * hkv * d
    raw = [torch.randint(-30000, 30000, (layers, n_blocks, block + pad), generator=g, dtype=width).to(DEV) for _ in range(2)]
    views = [r.view(dtype)[:, :, :block].as_strided((layers, n_blocks, bs, hkv, d),
                                                    (n_blocks * (block + pad), block + pad, hkv * d, d, 1)) for r in raw]
    return S.KVCache(*views), raw


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layers,bs,hkv,d,pad,pairs", [(1, 1, 1, 2, 0, 1), (2, 5, 1, 6, 2, 9), (3, 16, 8, 128, 0, 70), (2, 16, 2, 64, 8, 200),
                                                       (1, 24, 3, 80, 0, 3), (5, 64, 4, 128, 64, 20), (33, 7, 1, 64, 0, 65)])
def test_copies(layers, bs, hkv, d, pad, pairs, dtype):
    n = 2 * pairs + 3
    cache, raw = _pools(layers, n, bs, hkv, d, dtype, pairs, pad)
    rs = np.random.RandomState(pairs)
    ids = rs.permutation(n)
    src, dst, tokens = ids[:pairs].copy(), ids[pairs:2 * pairs].copy(), rs.randint(-2, bs + 3, size=pairs)
    for i in range(0, pairs, 4):  # some that are left out
        (src if i % 8 else dst)[i] = rs.choice([-1, -2 ** 31, n, 2 ** 31 - 1])
    for filled in (tokens, None):
        want = [r.clone() for r in raw]
        for w in want:
            for i in range(pairs):
                count = (bs if filled is None else min(max(int(filled[i]), 0), bs)) * hkv * d
                if 0 <= src[i] < n and 0 <= dst[i] < n:
                    w[:, dst[i], :count] = w[:, src[i], :count]
        S.kv_copy_blocks(cache, _i32(src), _i32(dst), None if filled is None else _i32(filled))
        torch.cuda.synchronize()
        assert torch.equal(raw[0], want[0]) and torch.equal(raw[1], want[1])


@pytest.mark.parametrize("there", [0, 1, 70])
def test_long_lists_with_few_pairs(there):
    """The moves of a compaction in room for many more: at the front, and all over."""
    cache, raw = _pools(2, 150, 16, 1, 64, torch.bfloat16, there)
    ids = np.random.RandomState(there).permutation(150)
    src, dst = np.full(70_000, -1), np.full(70_000, -1)
    at = np.arange(there) if there < 70 else np.random.RandomState(1).permutation(70_000)[:there]
    src[at], dst[at] = ids[:there], ids[there:2 * there]
    want = [r.clone() for r in raw]
    for w in want:
        w[:, ids[there:2 * there]] = w[:, ids[:there]]
    S.kv_copy_blocks(cache, _i32(src), _i32(dst))
    torch.cuda.synchronize()
    assert torch.equal(raw[0], want[0]) and torch.equal(raw[1], want[1])


def test_copies_behind_four_gigabytes():
    pool = lambda: torch.zeros((2, 70_000, 16, 8, 128), dtype=torch.bfloat16, device=DEV)  # noqa: E731
    cache = S.KVCache(pool(), pool())
    cache.k_pool[1, 69_999], cache.v_pool[1, 69_999] = 3.0, 5.0
    cache.k_pool[0, 1], cache.v_pool[1, 1] = 2.0, 4.0
    S.kv_copy_blocks(cache, _i32([69_999, 1]), _i32([3, 69_998]), _i32([16, 9]))
    torch.cuda.synchronize()
    assert bool((cache.k_pool[1, 3] == 3).all()) and bool((cache.v_pool[1, 3] == 5).all()) and bool((cache.k_pool[0, 3] == 0).all())
    assert bool((cache.k_pool[0, 69_998, :9] == 2).all()) and bool((cache.v_pool[1, 69_998, :9] == 4).all())
    assert bool((cache.v_pool[1, 69_998, 9:] == 0).all()) and bool((cache.k_pool[1, 69_998] == 0).all())
    assert float(cache.k_pool.sum(dtype=torch.float64)) == 16 * 1024 * (3 + 3 + 2) + 9 * 1024 * 2
