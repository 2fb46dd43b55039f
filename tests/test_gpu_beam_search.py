"""A search over the paged cache with all of its operators together, and the operators in graphs and on streams."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import beam_ref as R  # noqa: E402
import beam_search as E  # noqa: E402
import paper_2412_16434_amd as S  # noqa: E402

DEV = "cuda:0"


def test_the_host_side_of_a_search():
    state = E.Search([[1], [2]], beams=2, end=9)
    state.step([0, 0, 1, 1], [5, 6, 7, 8], [-1.0, -2.0, -1.0, -3.0], [-float("inf"), -4.0])
    assert state.histories == [[[5], [6]], [[7], [8]]] and state.ended == [[], [(-4.0, [9])]]
    state.step([1, 0, 2, 2], [3, 4, 9, 1], [-2.5, -2.75, -1.5, -9.0], [-1.0, -float("inf"), -1.25, -float("inf")])
    assert state.histories == [[[6, 3], [5, 4]], [[7, 9], [7, 1]]] and state.ended[0] == [(-0.5, [5, 9])]
    assert state.best() == [[5, 9], [7, 9]]


@pytest.mark.gpu
@pytest.mark.parametrize("block_size,sessions,beams,compact_every", [(16, 3, 4, 5), (5, 2, 3, 1), (1, 1, 2, 4), (16, 1, 1, 0), (4, 2, 7, 3)])
def test_the_cache_does_not_change_the_search(block_size, sessions, beams, compact_every):
    model = E.Scorer(layers=2)
    g = torch.Generator().manual_seed(sessions + beams)
    prompts = [torch.randint(0, 512, (9 + 4 * s,), generator=g).tolist() for s in range(sessions)]
    best, beams_, packed = E.search(model, prompts, beams, 12, 7, block_size, compact_every)
    plain, plain_beams = E.search_without_cache(model, prompts, beams, 12, 7)
    assert best == plain and beams_ == plain_beams
    assert len(packed) == (12 // compact_every if compact_every else 0)


@pytest.mark.gpu
def test_the_script_runs(capsys):
    assert E.main(["--sessions", "2", "--tokens", "8"]) == 0
    assert "2 of 2 sessions have the same best sequence" in capsys.readouterr().out
    assert E.main(["--sessions", "1", "--tokens", "6", "--dtype", "bf16"]) == 0


def _step_state(rs, sessions, beams, n_blocks, vocab, dtype, layers=2):
    """A step's inputs and outputs, and a function that makes its calls."""
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32).to(DEV).contiguous()  # noqa: E731
    z = lambda *n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    lens, held, table, refs, _ = R.shared_pages(rs, sessions, beams, 16, 200, n_blocks, ahead=0)
    rows = sessions * beams
    st = dict(logits=torch.zeros((rows, vocab), dtype=dtype, device=DEV), scores=torch.zeros(rows, device=DEV),
              cu=i32(np.arange(sessions + 1) * beams), lens=i32(lens), held=i32(held), table=i32(table), refs=i32(refs),
              parents=z(rows), tokens=z(rows), best=torch.zeros(rows, device=DEV), ends=torch.zeros(rows, device=DEV),
              refs1=z(n_blocks), free=z(n_blocks), n_free=z(1), table1=z(*table.shape), lens1=z(rows), held1=z(rows), refs2=z(n_blocks),
              src=z(rows), dst=z(rows), count=z(rows), taken=z(1), drop=z(rows), map=z(n_blocks), refs3=z(n_blocks), table2=z(*table.shape),
              msrc=z(n_blocks // 2), mdst=z(n_blocks // 2), counts=z(3))
    pool = lambda: torch.zeros((layers, n_blocks, 16, 1, 64), dtype=dtype, device=DEV)  # noqa: E731
    cache = S.KVCache(pool(), pool())
    st["k_pool"], st["v_pool"] = cache.k_pool, cache.v_pool
    space = torch.empty(S.beam_select_workspace_bytes(rows, vocab, beams), dtype=torch.uint8, device=DEV)
    space2 = torch.empty(S.kv_compact_workspace_bytes(n_blocks), dtype=torch.uint8, device=DEV)

    def fill(seed):
        g = torch.Generator().manual_seed(seed)
        st["logits"].copy_(torch.randn((rows, vocab), generator=g) * 3)
        st["scores"].copy_(-torch.rand(rows, generator=g) * 5)
        st["drop"].copy_((torch.rand(rows, generator=g) < 0.2).int())
        for p in (cache.k_pool, cache.v_pool):
            p.copy_(torch.randn(p.shape, generator=g))

    def run():
        S.beam_select(st["logits"], st["scores"], st["cu"], st["cu"], beams, st["parents"], st["tokens"], st["best"], end_token=5,
                      end_scores=st["ends"], workspace=space)
        S.kv_free(st["drop"], st["lens"], st["table"], st["refs"], 16, st["refs1"], st["free"], st["n_free"], held_blocks=st["held"],
                  workspace=space2)
        S.kv_free(None, None, None, st["refs"], 16, st["refs1"], st["free"], st["n_free"], workspace=space2)
        S.kv_fork(st["parents"], st["lens"], st["table"], st["refs1"], st["free"], 16, st["table1"], st["lens1"], st["refs2"], st["src"],
                  st["dst"], st["count"], held_blocks=st["held"], held_out=st["held1"], blocks_taken=st["taken"])
        S.kv_copy_blocks(cache, st["src"], st["dst"], st["count"])
        S.kv_compact(st["refs2"], -1, st["lens1"], st["table1"], 16, st["table2"], st["refs3"], st["map"], st["msrc"], st["mdst"],
                     st["counts"], held_blocks=st["held1"], workspace=space2)
        S.kv_copy_blocks(cache, st["msrc"], st["mdst"])
    return st, fill, run


@pytest.mark.gpu
@pytest.mark.parametrize("sessions,beams,n_blocks,vocab,dtype", [(2, 3, 400, 700, torch.float32), (30, 8, 20000, 40001, torch.bfloat16)])
def test_steps_in_a_graph(sessions, beams, n_blocks, vocab, dtype):
    """Captured once and replayed with other inputs, eager work between the replays: every replay is the eager call."""
    st, fill, run = _step_state(np.random.RandomState(2), sessions, beams, n_blocks, vocab, dtype)
    fill(0)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in (1, 2, 3, 4):
        fill(seed)
        run()
        want = {k: v.clone() for k, v in st.items()}
        fill(seed)
        for k, v in st.items():
            if k not in ("logits", "scores", "cu", "lens", "held", "table", "refs", "drop", "k_pool", "v_pool"):
                v.fill_(-3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        cols = torch.arange(st["table"].shape[1], device=DEV)
        inside = cols < st["held1"][:, None]
        for k, v in st.items():
            if k in ("table1", "table2"):   # (entries behind a row's blocks are left as they were)
                assert torch.equal(v[inside], want[k][inside]), k
                assert bool((v[~inside] == -3).all()), k
            else:
                assert torch.equal(v, want[k]), k


@pytest.mark.gpu
def test_calls_go_to_the_current_stream():
    """On a side stream: a delay, the inputs copied over other values, the calls.  Launched anywhere else they would not wait."""
    st, fill, run = _step_state(np.random.RandomState(6), 3, 4, 900, 5000, torch.float32)
    fill(1)
    run()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in st.items()}
    fill(1)
    logits, refs, lens = (st[k].clone() for k in ("logits", "refs", "lens"))
    st["logits"].fill_(1.0), st["refs"].fill_(1), st["lens"].fill_(3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        for k, v in (("logits", logits), ("refs", refs), ("lens", lens)):
            st[k].copy_(v)
        run()
    side.synchronize()
    for k, v in st.items():
        assert torch.equal(v, want[k]), k


@pytest.mark.gpu
def test_two_steps_at_once():
    """The same calls on two streams, each with its own inputs, outputs and workspaces."""
    steps = [_step_state(np.random.RandomState(s), 8, 4, 9000, 20001, torch.bfloat16) for s in (1, 2)]
    wants = []
    for seed, (st, fill, run) in enumerate(steps):
        fill(seed)
        run()
        torch.cuda.synchronize()
        wants.append({k: v.clone() for k, v in st.items()})
        fill(seed)
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for (st, fill, run), stream in zip(steps, streams):
        with torch.cuda.stream(stream):
            run()
    torch.cuda.synchronize()
    for (st, _, _), want in zip(steps, wants):
        for k, v in st.items():
            assert torch.equal(v, want[k]), k
