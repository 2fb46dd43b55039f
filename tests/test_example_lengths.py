"""The drafted step's example: what its host keeps of the sessions' lengths (the operators replaced; no GPU needed)."""
import os
import random
import sys
import types

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import drafted_steps as E  # noqa: E402


class Operators:
    """The package's calls as the server makes them; every session accepts what `accepted` says, and the bounds that the attention
    is called with are kept."""

    def __init__(self, accepted):
        self.accepted, self.bounds, self.queries = accepted, [], []

    KVCache = staticmethod(lambda k, v: types.SimpleNamespace(k_pool=k, v_pool=v))
    tree_mask = kv_commit = prefix_prefill_attn = staticmethod(lambda *a, **k: None)
    prefix_prefill_attn_workspace_bytes = staticmethod(lambda *a: 0)

    @staticmethod
    def build_tables(lens, new, table, free, bs, n_blocks, total, cu_new_lens, **outputs):
        cu_new_lens[1:] = torch.cumsum(new, 0)

    def tree_attn_workspace_bytes(self, cache, n, hq, total, most, longest):
        self.queries.append(longest)
        return 0

    def tree_attn(self, cache, layer, q, k, v, out, mask, cu, lens, table, most, longest, scale, workspace):
        self.bounds.append((longest, lens.tolist(), table.shape[1]))
        out.zero_()

    def tree_accept(self, draft, parents, target, cu, lens, rows, count, following, new_lens):
        sizes = (cu[1:] - cu[:-1]).tolist()
        count.copy_(torch.tensor([min(a, n) for a, n in zip(next(self.accepted), sizes)]))
        new_lens.copy_(lens + count)


@pytest.mark.parametrize("seed", range(3))
def test_the_longest_session_is_one_sessions_length(monkeypatch, seed):
    """Sessions that accept long paths in different steps: the sum of each step's longest path is no session's length."""
    rng, steps, n = random.Random(seed), 20, 4
    paths = [[rng.choice([1, 8]) for _ in range(n)] for _ in range(steps)]
    calls = Operators(iter(paths))
    monkeypatch.setattr(E, "S", calls)
    monkeypatch.setattr(E, "DEV", "cpu")
    model = E.Model(layers=1, hidden=32, n_q_heads=2, n_kv_heads=1, vocab=16)
    server = E.Server(model, n, 40 + 8 * steps)
    prompts = [list(range(k)) for k in (12, 9, 3, 1)]
    server.prompts([[t % 16 for t in p] for p in prompts])
    lens = [len(p) for p in prompts]
    for path in paths:
        sizes = [8] * (n - 1) + [rng.choice([0, 8])]
        server.step([([1] * k, [-1] + [0] * (k - 1) if k else []) for k in sizes])
        longest, on_device, stride = calls.bounds[-1]
        assert on_device == lens
        assert longest == calls.queries[-1] == max(lens) and longest <= stride * server.bs
        lens = [a + min(b, k) for a, b, k in zip(lens, path, sizes)]
    assert server.lens.tolist() == lens
