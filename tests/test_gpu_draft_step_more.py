"""The speculative step's attention where its arithmetic or its cuts reach their ends, and the whole step in a graph."""
import numpy as np
import pytest
import torch

import draft_ref as R
import paper_2412_16434_amd as S
from gpu_util import DEV
from test_gpu_draft_step import KINDS, Draft, cumulated, dev, random_parents

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("prefix,new", [([300], [20]), ([1500, 40], [5, 30])])
def test_values_near_the_largest_of_their_type(dtype, d, prefix, new):
    """Sums of a few hundred of them would overflow; their mean does not."""
    draft = Draft(prefix, new, dtype, d, sigma=0.1, seed=51)
    for name in ("v_pool", "v_new"):
        a = getattr(draft, name)
        sign = np.signbit(a.view(np.float32)) if dtype == "fp32" else (a >> 15).astype(bool)
        big = np.float32(2.9e38)
        if dtype == "fp32":
            setattr(draft, name, np.where(np.isnan(a), a, np.where(sign, -big, big)).astype(np.float32))
        else:
            bits = int(np.array([big], np.float32).view(np.uint32)[0] >> 16)
            nan = (a & 0x7FFF) > 0x7F80
            setattr(draft, name, np.where(nan, a, np.where(sign, bits | 0x8000, bits)).astype(a.dtype))
    assert np.isfinite(draft.check()).all()


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("sigma", [100.0, 2000.0])
def test_scores_of_thousands_and_millions(dtype, d, sigma):
    Draft([400, 0, 2100], [30, 5, 9], dtype, d, hkv=1, sigma=sigma, seed=52).check()


@pytest.mark.parametrize("dtype,d", KINDS)
def test_a_tile_in_many_parts(dtype, d):
    Draft([20011], [20], dtype, d, hkv=1, g=4, seed=53).check()
    Draft([9007], [3], dtype, d, hkv=1, g=2, seed=54).check()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("g", [4, 1])
def test_ragged_sessions_beyond_a_waves_lanes(dtype, d, g):
    rng = np.random.default_rng(55)
    prefix, new = rng.integers(0, 300, 131), rng.integers(0, 30, 131)
    prefix[[5, 70, 130]], new[[0, 64, 128]] = [4000, 2500, 1800], 0
    Draft(prefix, new, dtype, d, hkv=1, g=g, tree="bits", seed=55).check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
def test_a_graph_of_the_step_follows_its_inputs(dtype, d):
    """Captured once, replayed on other lengths, trees and values, with eager work between the replays."""
    hkv, g, bs, layers, n, top, far, n_blocks = 2, 4, 16, 2, 5, 24, 900, 400
    torch_type = torch.bfloat16 if dtype == "bf16" else torch.float32
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)  # noqa: E731
    pools = [torch.randn((layers, n_blocks, bs, hkv, d), device=DEV).to(torch_type) for _ in range(2)]
    cache, total = S.KVCache(*pools), n * top
    lens, new, held, begin, parents, draft, target = i32(n), i32(n), i32(n), i32(1), i32(total), i32(total), i32(total)
    free = torch.randperm(n_blocks, device=DEV).int()
    first_table = torch.full((n, 60), -1, dtype=torch.int32, device=DEV)
    q = torch.empty((total, hkv * g, d), dtype=torch_type, device=DEV)
    k_new, v_new = (torch.empty((layers, total, hkv, d), dtype=torch_type, device=DEV) for _ in range(2))
    ws = torch.empty(S.tree_attn_workspace_bytes(cache, n, hkv * g, total, top, far), dtype=torch.uint8, device=DEV)
    written = dict(table=first_table.clone(), cu=i32(n + 1), slots=torch.zeros(total, dtype=torch.int64, device=DEV), positions=i32(total),
                   taken=i32(1), mask=torch.zeros((total, 1), dtype=torch.int64, device=DEV), out=torch.zeros_like(q), rows=i32(total),
                   count=i32(n), following=i32(n), after=i32(n))

    def step():
        w = written
        S.build_tables(lens, new, w["table"], free, bs, n_blocks, total, cu_new_lens=w["cu"], slot_map=w["slots"],
                       blocks_taken=w["taken"], held_blocks=held, free_begin=begin)
        S.tree_mask(parents, w["cu"], top, w["mask"], prefix_lens=lens, positions=w["positions"])
        S.tree_attn(cache, 1, q, k_new[1], v_new[1], w["out"], w["mask"], w["cu"], lens, w["table"], top, far, d ** -0.5, ws)
        S.tree_accept(draft, parents, target, w["cu"], lens, w["rows"], w["count"], w["following"], w["after"])
        S.kv_commit(cache, k_new, v_new, w["rows"], w["slots"])

    def fill(seed):
        rng = np.random.default_rng(seed)
        p, m = rng.integers(0, far, n), rng.integers(1, top + 1, n)
        have = -(-p // bs)
        table = np.full((n, 60), -1, np.int32)
        ids, at = free.cpu().numpy(), 0
        for s, k in enumerate(have):
            table[s, :k] = ids[at:at + k]
            at += int(k)
        lens.copy_(dev(p, np.int32)), new.copy_(dev(m, np.int32)), held.copy_(dev(have, np.int32)), begin.fill_(at)
        written["table"].copy_(dev(table))
        tree = np.concatenate([random_parents(int(k), rng, 4) for k in m])
        parents[:len(tree)].copy_(dev(tree))
        draft.copy_(dev(rng.integers(0, 3, total), np.int32)), target.copy_(dev(rng.integers(0, 3, total), np.int32))
        g_ = torch.Generator(DEV).manual_seed(seed)
        for t in (q, k_new, v_new):
            t.copy_(torch.randn(t.shape, generator=g_, device=DEV).to(torch_type))
        for name, t in written.items():
            if name != "table":
                t.zero_()

    fill(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    start = [p.clone() for p in pools]
    for seed in (1, 2, 3):
        results = []
        for run in (step, graph.replay):
            fill(seed)
            for p, was in zip(pools, start):
                p.copy_(was)
            run()
            torch.cuda.synchronize()
            m = int(written["cu"][-1])
            results.append([t.clone() if name not in ("out", "rows") else t[:m].clone() for name, t in written.items()] +
                           [p.clone() for p in pools])
        assert all(torch.equal(a, b) for a, b in zip(*results)), seed
        assert bool(results[0][6].float().abs().sum() > 0) and not torch.equal(results[0][-1], start[1])
        # and the commit put the accepted rows where the tables say
        cu, rows, slots = (written[k].cpu().numpy() for k in ("cu", "rows", "slots"))
        for s in range(n):
            path = R.accept(*(t[cu[s]:cu[s + 1]].cpu().numpy() for t in (draft, parents, target)))
            assert rows[cu[s]:cu[s] + len(path)].tolist() == [cu[s] + i for i in path]
            for k, i in enumerate(path):
                slot = int(slots[cu[s] + k])
                assert torch.equal(pools[0][:, slot // bs, slot % bs], k_new[:, cu[s] + i])


def test_a_session_before_any_token_and_an_empty_batch():
    empty = torch.zeros(0, dtype=torch.int32, device=DEV)
    cu = dev(cumulated([]))
    out = torch.zeros((0, 8, 128), dtype=torch.bfloat16, device=DEV)
    kv = torch.zeros((0, 2, 128), dtype=torch.bfloat16, device=DEV)
    pool = torch.zeros((1, 4, 16, 2, 128), dtype=torch.bfloat16, device=DEV)
    cache = S.KVCache(pool, pool.clone())
    mask = torch.zeros((0, 1), dtype=torch.int64, device=DEV)
    S.tree_mask(empty, cu, 0, mask)
    S.tree_attn(cache, 0, out, kv, kv, out, mask, cu, empty, torch.zeros((0, 1), dtype=torch.int32, device=DEV), 0, 0, 0.1)
    S.tree_accept(empty, empty, empty, cu, empty, empty, empty, empty)
    S.kv_commit(cache, kv[None], kv[None], empty, torch.zeros(0, dtype=torch.int64, device=DEV))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("sessions,g,long", [(64, 2, 0), (65, 2, 900), (256, 1, 0), (257, 4, 0), (300, 1, 1500), (600, 2, 0), (257, 16, 700)])
def test_numbers_of_sessions_around_a_waves_shares(dtype, d, sessions, g, long):
    """A lane has one session, or four, or four of every 256: empty ones at the edges, tiles of several sessions in a range."""
    rng = np.random.default_rng(sessions)
    prefix, new = rng.integers(0, 40, sessions), rng.integers(0, 6, sessions)
    new[[0, 63, sessions - 1]], prefix[sessions // 2], new[sessions // 2] = [0, 0, 4], max(long, 50), 5
    Draft(prefix, new, dtype, d, hkv=1, g=g, tree="bits", seed=61).check()
