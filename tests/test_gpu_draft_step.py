"""The speculative step's operators on the GPU against plain references in 64 bits: block tables and slot maps, tree masks,
the accepted path and its commit bit for bit; tree attention within bounds that follow from its arithmetic."""
import numpy as np
import pytest
import torch

import draft_ref as R
import paper_2412_16434_amd as S
import workloads as W
from gpu_util import DEV, to_dev, to_host, widen

pytestmark = pytest.mark.gpu


def dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a if dtype is None else np.asarray(a, dtype=dtype))).to(DEV)


def cumulated(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


# ------------------------------------------------------------------------------------------------------------------
# block tables and slot maps
# ------------------------------------------------------------------------------------------------------------------
def run_tables(prefix, new, table, free, bs, n_blocks, total, held=None, free_begin=None):
    n = len(prefix)
    got = dict(table=dev(table), cu=torch.full((n + 1,), 77, dtype=torch.int32, device=DEV),
               offsets=torch.full((n + 1,), 77, dtype=torch.int64, device=DEV),
               slots=torch.full((total,), 77, dtype=torch.int64, device=DEV),
               positions=torch.full((total,), 77, dtype=torch.int32, device=DEV),
               taken=torch.full((1,), 77, dtype=torch.int32, device=DEV),
               held_after=torch.full((n,), 77, dtype=torch.int32, device=DEV))
    S.build_tables(dev(prefix, np.int32), dev(new, np.int32), got["table"], dev(free, np.int32), bs, n_blocks, total,
                   cu_new_lens=got["cu"], token_offsets=got["offsets"], slot_map=got["slots"], positions=got["positions"],
                   blocks_taken=got["taken"], held_after=got["held_after"],
                   held_blocks=None if held is None else dev(held, np.int32),
                   free_begin=None if free_begin is None else dev([free_begin], np.int32))
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in got.items()}


def check_tables(prefix, new, bs, seed, short=0, held=None, free_begin=None, stride=None, total=None, bad_ids=False):
    rng = np.random.default_rng(seed)
    prefix, new = np.asarray(prefix), np.asarray(new)
    p, n = np.maximum(prefix, 0), np.maximum(new, 0)
    have = np.maximum(-(-p // bs), 0 if held is None else held)
    all_blocks = np.maximum(-(-(p + n) // bs), have)
    n_blocks = int(all_blocks.sum()) + 5
    perm = rng.permutation(n_blocks).astype(np.int32)
    table = np.full((len(p), max(int(all_blocks.max()) + 2, 1) if stride is None else stride), -9, np.int32)
    at = 0
    for s, k in enumerate(have):
        k = min(k, table.shape[1])
        table[s, :k] = perm[at:at + k]
        at += int(k)
    if bad_ids:
        table[::2, :1] = n_blocks + 3
        table[1::3, :1] = -2
    free = perm[at:] if short == 0 else perm[at:at + max(int((all_blocks - have).sum()) - short, 0)]
    total = int(n.sum()) if total is None else total
    want = R.build_tables(prefix, new, table, free, bs, n_blocks, total, held, free_begin or 0)
    got = run_tables(prefix, new, table, free, bs, n_blocks, total, held, free_begin)
    for k in want:
        assert np.array_equal(got[k], want[k]), f"{k}: {np.flatnonzero(got[k].ravel() != want[k].ravel())[:5]}"


@pytest.mark.parametrize("bs", [1, 7, 16, 64])
@pytest.mark.parametrize("sessions,p_hi,n_hi", [(1, 0, 1), (1, 300, 40), (5, 100, 1), (64, 500, 64), (1030, 70, 9), (2500, 33, 3)])
def test_tables_match_the_reference(bs, sessions, p_hi, n_hi):
    rng = np.random.default_rng(sessions * 7 + bs)
    check_tables(rng.integers(0, p_hi + 1, sessions), rng.integers(0, n_hi + 1, sessions), bs, 1)


def test_tables_of_arriving_sessions_and_long_turns():
    check_tables([0, 0, 0, 0], [5000, 0, 1, 2049], 16, 2)
    check_tables([0] * 40, list(range(100, 140)), 16, 3)
    check_tables([15, 16, 17, 0], [1, 1, 1, 16], 16, 4)


def test_tables_when_the_free_list_or_a_row_ends():
    check_tables([10, 20, 30, 0], [40, 40, 0, 70], 16, 5, short=3)
    check_tables([0, 0], [50, 50], 16, 6, short=100)          # an empty list
    check_tables([100, 3], [50, 60], 16, 7, stride=4)         # rows narrower than the sessions
    check_tables([40, 41, 42, 43, 44, 45], [3] * 6, 64, 8, bad_ids=True)


def test_tables_with_held_blocks_and_a_cursor():
    check_tables([33, 10, 0, 64], [20, 4, 5, 1], 16, 9, held=np.array([5, 1, 1, 3]), free_begin=2)
    check_tables([33, 10], [20, 4], 16, 10, free_begin=-1)     # no entry before the list
    check_tables([33, 10], [200, 4], 16, 11, free_begin=1 << 30)


def test_tables_with_an_understated_or_overstated_total_and_negative_lengths():
    check_tables([10, 20, 30], [40, 41, 42], 16, 12, total=70)
    check_tables([10, 20, 30], [40, 41, 42], 16, 13, total=1500)
    check_tables([-5, 20, -1], [4, -3, 6], 16, 14)


def test_tables_over_two_steps_use_the_blocks_of_what_was_not_accepted():
    bs, new = 4, np.array([6, 6], np.int32)
    prefix, table, free = np.array([3, 8], np.int32), np.full((2, 8), -1, np.int32), np.arange(10, 22, dtype=np.int32)
    table[0, 0], table[1, :2] = 1, [2, 3]
    one = run_tables(prefix, new, table, free, bs, 32, 12, held=np.array([1, 2], np.int32), free_begin=0)
    after = prefix + np.array([2, 1], np.int32)               # two tokens and one accepted
    two = run_tables(after, new, one["table"], free, bs, 32, 12, held=one["held_after"], free_begin=int(one["taken"][0]))
    owned = [set(two["table"][s, :two["held_after"][s]].tolist()) for s in range(2)]
    assert not owned[0] & owned[1] and all(-1 not in o for o in owned)
    assert np.array_equal(two["table"][0, :one["held_after"][0]], one["table"][0, :one["held_after"][0]])
    assert two["taken"][0] == len(owned[0]) + len(owned[1]) - 3


# ------------------------------------------------------------------------------------------------------------------
# masks of trees
# ------------------------------------------------------------------------------------------------------------------
def random_parents(n, rng, reach):
    return np.array([-1] + [int(rng.integers(max(0, i - reach), i)) for i in range(1, n)], np.int32)[:n]


def check_mask(parents, words=None, prefix=None, max_new=None):
    n = [len(p) for p in parents]
    total, top = sum(n), max(n)
    words = -(-top // 64) if words is None else words
    sees = [R.ancestors(p) for p in parents]
    mask = torch.full((total, words), 0x55, dtype=torch.int64, device=DEV)
    positions = torch.full((total,), 77, dtype=torch.int32, device=DEV)
    S.tree_mask(dev(np.concatenate(parents), np.int32), dev(cumulated(n)), top if max_new is None else max_new, mask,
                prefix_lens=None if prefix is None else dev(prefix, np.int32), positions=positions)
    torch.cuda.synchronize()
    assert np.array_equal(mask.cpu().numpy(), R.pack_bits(sees, words))
    base = np.repeat(np.zeros(len(n), np.int64) if prefix is None else prefix, n)
    assert np.array_equal(positions.cpu().numpy(), base + np.concatenate([s.sum(axis=1) - 1 for s in sees]))


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 128, 200, 257, 1000])
@pytest.mark.parametrize("reach", [1, 5, 100])
def test_masks_match_the_reference(n, reach):
    rng = np.random.default_rng(n + reach)
    check_mask([random_parents(n, rng, reach)], prefix=[13])


def test_masks_of_many_sessions_with_empty_ones():
    rng = np.random.default_rng(1)
    sizes = [0, 1, 64, 0, 65, 7, 130, 0]
    check_mask([random_parents(k, rng, 9) for k in sizes], prefix=rng.integers(0, 1000, len(sizes)))
    check_mask([random_parents(int(k), rng, 4) for k in rng.integers(1, 40, 300)])


def test_masks_of_forests_bad_parents_and_wide_rows():
    check_mask([np.array([-1, -1, 0, 1, -1, 4], np.int32), np.array([5, 0, 7, 2, -8, 4, 6], np.int32)], words=3, prefix=[4, 0])
    check_mask([np.array([0, 1, 2, 3], np.int32)])              # a node that names itself or a later one is a root
    check_mask([np.arange(-1, 99, dtype=np.int32)], max_new=100)


def test_mask_of_the_largest_tree():
    rng = np.random.default_rng(3)
    check_mask([random_parents(4096, rng, 60)])


# ------------------------------------------------------------------------------------------------------------------
# accepted path and commit
# ------------------------------------------------------------------------------------------------------------------
def random_draft(n, rng, vocab):
    return rng.integers(0, vocab, n).astype(np.int32), random_parents(n, rng, 5), rng.integers(0, vocab, n).astype(np.int32)


@pytest.mark.parametrize("sizes", [[1], [0, 3, 0], [64, 65, 1, 0, 130], [300], list(range(1, 90))])
@pytest.mark.parametrize("vocab", [1, 2, 5])
def test_accepted_paths_match_the_reference(sizes, vocab):
    rng = np.random.default_rng(sum(sizes) + vocab)
    trees = [random_draft(k, rng, vocab) for k in sizes]
    cu, total = cumulated(sizes), sum(sizes)
    prefix = rng.integers(0, 1000, len(sizes)).astype(np.int32)
    rows, counts, nxt = np.full(total, -1), [], []
    for first, (draft, parents, target) in zip(cu, trees):
        path = R.accept(draft, parents, target)
        rows[first:first + len(path)] = first + np.array(path, dtype=np.int64)
        counts.append(len(path))
        nxt.append(target[path[-1]] if path else -1)
    e = lambda k: torch.full((k,), 77, dtype=torch.int32, device=DEV)  # noqa: E731
    got_rows, got_counts, got_next, lens = e(total), e(len(sizes)), e(len(sizes)), dev(prefix)
    flat = [dev(np.concatenate([t[i] for t in trees]), np.int32) for i in range(3)]
    S.tree_accept(flat[0], flat[1], flat[2], dev(cu), lens, got_rows, got_counts, got_next, new_prefix_lens=lens)  # in place
    torch.cuda.synchronize()
    assert np.array_equal(got_rows.cpu().numpy(), rows)
    assert got_counts.tolist() == counts and got_next.tolist() == nxt
    assert np.array_equal(lens.cpu().numpy(), prefix + np.array(counts))


def test_a_parent_behind_its_child_is_no_parent():
    one = torch.zeros(4, dtype=torch.int32, device=DEV)
    rows, count, nxt = one.clone(), one[:1].clone(), one[:1].clone()
    # nodes 1 and 2 name each other, node 3 itself: all tokens agree, only the root is accepted
    S.tree_accept(one, dev([-1, 2, 1, 3], np.int32), one, dev([0, 4], np.int32), None, rows, count, nxt)
    assert rows.tolist() == [0, -1, -1, -1] and count.tolist() == [1] and nxt.tolist() == [0]


@pytest.mark.parametrize("dtype,layers,hkv,d,bs,strided", [
    ("bf16", 3, 8, 128, 16, False), ("bf16", 2, 2, 64, 7, True), ("fp32", 1, 3, 20, 4, False), ("bf16", 5, 1, 6, 1, False),
    ("fp32", 2, 2, 128, 32, True)])
def test_commit_writes_the_named_rows_and_nothing_else(dtype, layers, hkv, d, bs, strided):
    rng = np.random.default_rng(layers * 100 + d)
    n_blocks, n_rows, n_entries = 40, 90, 150
    shape = (layers, n_blocks * (2 if strided else 1), bs, hkv, d)
    ints = torch.int16 if dtype == "bf16" else torch.int32
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    draw = lambda shp: torch.from_numpy(rng.integers(-30000, 30000, shp).astype(np.int16 if ints == torch.int16 else np.int32))  # noqa: E731
    k_all, v_all, k_new, v_new = draw(shape), draw(shape), draw((layers, n_rows, hkv, d)), draw((layers, n_rows, hkv, d))
    rows = rng.integers(-1, n_rows + 5, n_entries).astype(np.int32)
    slots = rng.permutation(n_blocks * bs + 200)[:n_entries].astype(np.int64) - 20
    slots[0], slots[1] = (1 << 62) + 5, -(1 << 62)
    kd, vd = k_all.to(DEV), v_all.to(DEV)
    view = (lambda t: t.view(tt)[:, ::2]) if strided else (lambda t: t.view(tt))
    S.kv_commit(S.KVCache(view(kd), view(vd)), k_new.to(DEV).view(tt), v_new.to(DEV).view(tt), dev(rows), dev(slots))
    torch.cuda.synchronize()
    for t, slot in zip(rows, slots):
        if 0 <= t < n_rows and 0 <= slot < n_blocks * bs:
            b = slot // bs * (2 if strided else 1)
            k_all[:, b, slot % bs], v_all[:, b, slot % bs] = k_new[:, t], v_new[:, t]
    assert torch.equal(kd.cpu(), k_all) and torch.equal(vd.cpu(), v_all)


# ------------------------------------------------------------------------------------------------------------------
# tree attention
# ------------------------------------------------------------------------------------------------------------------
class Draft:
    """Seeded host inputs of one call; every pool slot that no session owns holds NaN."""

    def __init__(self, prefix, new, dtype="bf16", d=128, hkv=2, g=4, bs=16, tree="tree", sigma=1.0, seed=0, layers=1):
        rng = np.random.default_rng(seed)
        self.prefix, self.new, self.dtype, self.bs, self.scale = np.array(prefix, np.int32), list(new), dtype, bs, 1 / np.sqrt(d)
        total, need = sum(new), [-(-p // bs) for p in prefix]
        n_blocks = sum(need) + 3
        perm, at = rng.permutation(n_blocks), 0
        self.table = np.full((len(prefix), max(max(need), 1)), -1, np.int32)
        cast = W.f32_to_bf16_bits if dtype == "bf16" else (lambda a: a)
        normal = lambda shape: rng.standard_normal(shape).astype(np.float32) * np.float32(sigma)  # noqa: E731
        k, v = (np.full((n_blocks, bs, hkv, d), np.nan, np.float32) for _ in range(2))
        for s, p in enumerate(prefix):
            ids = perm[at:at + need[s]]
            self.table[s, :need[s]] = ids
            at += need[s]
            for j, b in enumerate(ids):
                rows = min(bs, p - j * bs)
                k[b, :rows], v[b, :rows] = normal((rows, hkv, d)), normal((rows, hkv, d))
        self.k_pool, self.v_pool = cast(k), cast(v)
        self.q, self.k_new, self.v_new = (cast(normal((total, h, d))) for h in (hkv * g, hkv, hkv))
        self.cu = cumulated(new)
        if tree == "tree":
            self.sees = [R.ancestors(random_parents(n, rng, 4)) for n in new]
        elif tree == "causal":
            self.sees = [np.tril(np.ones((n, n), bool)) for n in new]
        elif tree == "none":
            self.sees = [np.zeros((n, n), bool) for n in new]
        else:
            self.sees = [(rng.random((n, n)) < 0.3) & (rng.random((n, 1)) < 0.7) for n in new]
        self.words = -(-max(max(new), 1) // 64)

    def mask(self):
        return R.pack_bits(self.sees, self.words)

    def run(self, max_new=None, max_prefix=None, alias=False, shift=0, stream=None, out=None):
        kp, vp = to_dev(self.k_pool)[None], to_dev(self.v_pool)[None]
        q, kn, vn = to_dev(self.q), to_dev(self.k_new), to_dev(self.v_new)
        if shift:  # the same values, not on 16 bytes
            moved = torch.empty(q.numel() + shift, dtype=q.dtype, device=DEV)[shift:].view(q.shape)
            moved.copy_(q)
            q = moved
        out = q if alias else torch.full_like(q, float("nan"))
        cache = S.KVCache(kp, vp)
        top = max(self.new) if max_new is None else max_new
        far = int(self.prefix.max()) if max_prefix is None else max_prefix
        size = S.tree_attn_workspace_bytes(cache, len(self.prefix), q.shape[1], q.shape[0], top, far)
        ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) if size else None
        S.tree_attn(cache, 0, q, kn, vn, out, dev(self.mask()), dev(self.cu), dev(self.prefix), dev(self.table), top, far,
                    float(self.scale), workspace=ws)
        torch.cuda.synchronize()
        return widen(to_host(out))

    def reference(self):
        return R.tree_attn(*(widen(a) for a in (self.k_pool, self.v_pool, self.q, self.k_new, self.v_new)), self.sees, self.cu,
                           self.prefix, self.table, float(np.float32(self.scale)))

    def check(self, **kw):
        got = self.run(**kw)
        ref, weight, spread = self.reference()
        keys, d = int(self.prefix.max()) + max(self.new), self.q.shape[2]
        assert np.array_equal(np.isnan(got), np.isnan(ref)), "NaN in other places"
        fine = np.isfinite(ref)
        assert np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)])
        with np.errstate(invalid="ignore"):
            off = np.abs(got - ref)
        # What 32-bit arithmetic may cost: a score is a sum of d products (relative to the sum of their magnitudes), an
        # exponential has that error of its argument, numerator and denominator are sums of `keys` terms.
        u = 2.0 ** -24
        part = 2 * (d + 4) * u * spread + 2 * (keys + 16) * u
        if self.dtype == "bf16":  # probabilities keep 16 bits, the output is rounded to 8
            allowed = 2.0 ** -8 * np.abs(ref) + (part[..., None] + 2.0 ** -14) * weight
        else:
            allowed = part[..., None] * weight + 2 * u * np.abs(ref)
        with np.errstate(invalid="ignore"):
            worst = np.where(fine, off - allowed, -1.0)
        assert worst.max() <= 0, f"off by {off[np.unravel_index(worst.argmax(), worst.shape)]} at {np.unravel_index(worst.argmax(), worst.shape)}"
        norm = np.sqrt((ref[fine] ** 2).sum())
        if norm > 0:  # rounding to 8 bits is at most 2^-8 / sqrt(3) in the 2-norm
            rel = np.sqrt((off[fine] ** 2).sum()) / norm
            assert rel <= (2.6e-3 if self.dtype == "bf16" else 2e-6), rel
        return got


KINDS = [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)]


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("prefix,new", [
    ([0], [1]), ([1], [1]), ([31, 32, 33], [1, 2, 3]), ([256], [8]), ([700], [26]), ([0, 5, 90], [64, 65, 40]),
    ([100, 0, 17], [0, 9, 0]), ([1200, 3], [7, 130])])
def test_trees_of_every_size(dtype, d, prefix, new):
    Draft(prefix, new, dtype, d, seed=1).check()


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("hkv,g", [(1, 1), (3, 7), (8, 4), (2, 16), (1, 5), (2, 33)])
def test_heads_and_groups(dtype, d, hkv, g):
    Draft([70, 300], [6, 11], dtype, d, hkv=hkv, g=g, seed=2).check()


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("bs", [1, 3, 8, 16, 24, 64, 256])
def test_block_sizes(dtype, d, bs):
    Draft([0, 63, 64, 277], [5, 17, 1, 9], dtype, d, bs=bs, seed=3).check()


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("tree", ["bits", "causal", "none"])
def test_masks_that_are_no_trees_and_rows_that_see_nothing(dtype, d, tree):
    draft = Draft([0, 40, 0, 513], [12, 70, 1, 20], dtype, d, tree=tree, seed=4)
    got = draft.check()
    for s, P in enumerate(draft.prefix):
        if P == 0:
            empty = ~draft.sees[s].any(axis=1)
            assert np.all(got[draft.cu[s]:draft.cu[s + 1]][empty] == 0)


@pytest.mark.parametrize("dtype,d", KINDS)
def test_long_prefixes_are_cut_and_joined(dtype, d):
    Draft([5000, 1, 2111], [9, 4, 33], dtype, d, hkv=1, g=4, seed=5).check()


def test_more_sessions_than_lanes():
    rng = np.random.default_rng(6)
    Draft(rng.integers(0, 90, 150), rng.integers(0, 5, 150), hkv=1, g=2, d=64, seed=6).check()
    Draft(np.where(np.arange(70) == 68, 3000, 10), np.full(70, 3), hkv=1, g=4, seed=7).check()


@pytest.mark.parametrize("dtype,d", KINDS)
def test_bounds_that_are_too_low_or_too_high_change_no_result(dtype, d):
    draft = Draft([900, 1500, 0], [20, 3, 40], dtype, d, hkv=1, seed=8)
    draft.check(max_new=1, max_prefix=1)
    draft.check(max_prefix=int(draft.table.shape[1] * draft.bs))
    draft.check(max_new=60)


@pytest.mark.parametrize("dtype,d", KINDS)
def test_addresses_that_are_not_on_16_bytes(dtype, d):
    Draft([200, 0, 33], [5, 9, 1], dtype, d, tree="bits", seed=9).check(shift=1)


@pytest.mark.parametrize("dtype,d", KINDS)
def test_the_output_may_be_the_query(dtype, d):
    Draft([1500, 40], [33, 70], dtype, d, seed=10).check(alias=True)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("sigma", [1e-3, 8.0])
def test_flat_and_sharp_softmax(dtype, d, sigma):
    Draft([600, 20], [17, 5], dtype, d, sigma=sigma, seed=11).check()


def put(draft, where, index, value):
    a = getattr(draft, where)
    a[index] = value if draft.dtype == "fp32" else W.f32_to_bf16_bits(np.array([value], np.float32))[0]


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf, 3.3e38])
def test_masked_tokens_may_hold_anything(dtype, d, value):
    draft = Draft([70, 0, 1300], [9, 40, 70], dtype, d, tree="bits", seed=12)
    for s, j in ((0, 3), (1, 17), (2, 66)):       # hidden from all others, and from itself where the row is not empty
        draft.sees[s][:, j] = False
        put(draft, "v_new", (draft.cu[s] + j, 1), value)
        put(draft, "k_new", (draft.cu[s] + j, 1), value if not np.isfinite(value) else 1e30)  # (1e30: its products still fit)
    draft.sees[1][5, 17] = True                    # one row does see it
    draft.check()


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("where", ["v_pool", "k_pool", "q"])
def test_infinities_and_nan_that_are_seen(dtype, d, value, where):
    draft = Draft([900, 30], [5, 3], dtype, d, hkv=1, seed=13)
    if where == "q":
        put(draft, "q", (2, 1, 7), value)
    else:
        put(draft, where, (draft.table[0, 3], 5, 0, 11), value)
    draft.check()


@pytest.mark.parametrize("dtype,d", KINDS)
def test_block_ids_outside_the_cache_are_rows_of_zeros(dtype, d):
    draft = Draft([300, 45], [6, 6], dtype, d, seed=14)
    draft.table[0, 2], draft.table[0, 7], draft.table[1, 0] = -5, 1 << 30, draft.k_pool.shape[0]
    draft.check()


def test_offsets_past_32_bits():
    draft = Draft([500], [12], hkv=8, g=4, seed=15)
    n_blocks = 150000                              # 150000 * 16 * 1024 elements: 2.4e9
    pools = [torch.zeros((1, n_blocks, 16, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    table = draft.table.copy()
    for j in range(table.shape[1]):
        for pool, host in zip(pools, (draft.k_pool, draft.v_pool)):
            pool[0, n_blocks - 1 - 2 * j] = to_dev(host[table[0, j]])
        draft.table[0, j] = n_blocks - 1 - 2 * j
    cache = S.KVCache(*pools)
    q, out = to_dev(draft.q), torch.empty(draft.q.shape, dtype=torch.bfloat16, device=DEV)
    size = S.tree_attn_workspace_bytes(cache, 1, 32, 12, 12, 500)
    S.tree_attn(cache, 0, q, to_dev(draft.k_new), to_dev(draft.v_new), out, dev(draft.mask()), dev(draft.cu), dev(draft.prefix),
                dev(draft.table), 12, 500, float(draft.scale),
                workspace=torch.empty(size, dtype=torch.uint8, device=DEV) if size else None)
    torch.cuda.synchronize()
    draft.table = table
    assert np.array_equal(widen(to_host(out)), draft.run())


def test_layers_and_strides_of_the_cache():
    draft = Draft([130, 40], [7, 20], seed=16)
    wide = [torch.full((3, draft.k_pool.shape[0], 2, *draft.k_pool.shape[1:]), float("nan"), dtype=torch.bfloat16, device=DEV)
            for _ in range(2)]
    for t, host in zip(wide, (draft.k_pool, draft.v_pool)):
        t[2, :, 0] = to_dev(host)
    cache = S.KVCache(*(t[:, :, 0] for t in wide))  # every other block, layer 2
    q, out = to_dev(draft.q), torch.empty(draft.q.shape, dtype=torch.bfloat16, device=DEV)
    S.tree_attn(cache, 2, q, to_dev(draft.k_new), to_dev(draft.v_new), out, dev(draft.mask()), dev(draft.cu), dev(draft.prefix),
                dev(draft.table), 20, 130, float(draft.scale),
                workspace=torch.empty(1 << 20, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    assert np.array_equal(widen(to_host(out)), draft.run())


def test_a_causal_mask_is_the_prefill_attention():
    draft = Draft([333, 0, 64], [40, 17, 1], tree="causal", seed=17)
    got = draft.run()
    cache = S.KVCache(to_dev(draft.k_pool)[None], to_dev(draft.v_pool)[None])
    q, out = to_dev(draft.q), torch.empty(draft.q.shape, dtype=torch.bfloat16, device=DEV)
    args = (len(draft.prefix), q.shape[1], q.shape[0], 40, 333)
    size = S.prefix_prefill_attn_workspace_bytes(cache, *args)
    S.prefix_prefill_attn(cache, 0, q, to_dev(draft.k_new), to_dev(draft.v_new), out, dev(draft.cu), dev(draft.prefix),
                          dev(draft.table), 40, 333, float(draft.scale),
                          workspace=torch.empty(size, dtype=torch.uint8, device=DEV) if size else None)
    torch.cuda.synchronize()
    other = widen(to_host(out))
    # two roundings of the output to 8 bits, and the other call's probabilities with 8 bits
    assert np.sqrt(((got - other) ** 2).sum() / (other ** 2).sum()) <= 3 * 2.0 ** -8 / np.sqrt(3)


def test_a_workspace_that_is_too_small_is_refused():
    draft = Draft([5000], [9], hkv=1, seed=18)
    cache = S.KVCache(to_dev(draft.k_pool)[None], to_dev(draft.v_pool)[None])
    q = to_dev(draft.q)
    args = (cache, 0, q, to_dev(draft.k_new), to_dev(draft.v_new), torch.empty_like(q), dev(draft.mask()), dev(draft.cu),
            dev(draft.prefix), dev(draft.table), 9, 5000, float(draft.scale))
    size = S.tree_attn_workspace_bytes(cache, 1, q.shape[1], 9, 9, 5000)
    assert size > 0
    for ws in (None, torch.empty(size - 1, dtype=torch.uint8, device=DEV)):
        with pytest.raises(S.SymphError) as e:
            S.tree_attn(*args, workspace=ws)
        assert e.value.status == -4


def test_calls_on_another_stream_and_in_a_graph():
    draft = Draft([2500, 77], [9, 40], hkv=2, seed=19)
    want = draft.run()
    cache = S.KVCache(to_dev(draft.k_pool)[None], to_dev(draft.v_pool)[None])
    q, out = to_dev(draft.q), torch.empty(draft.q.shape, dtype=torch.bfloat16, device=DEV)
    size = S.tree_attn_workspace_bytes(cache, 2, q.shape[1], q.shape[0], 40, 2500)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
    args = (cache, 0, q, to_dev(draft.k_new), to_dev(draft.v_new), out, dev(draft.mask()), dev(draft.cu), dev(draft.prefix),
            dev(draft.table), 40, 2500, float(draft.scale))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        S.tree_attn(*args, workspace=ws)
    side.synchronize()
    assert np.array_equal(widen(to_host(out)), want)
    out.zero_()
    torch.cuda.synchronize()
    S.tree_attn(*args, workspace=ws, stream=side)  # named, not current
    side.synchronize()
    assert np.array_equal(widen(to_host(out)), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.tree_attn(*args, workspace=ws)
    for _ in range(3):
        out.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(widen(to_host(out)), want)
