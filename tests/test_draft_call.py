"""The compiled marshalling of the drafted step's calls against the general path: it takes the same calls with the same results,
and leaves everything it does not take, errors above all, to the general path."""
import pytest
import torch

import paper_2412_16434_amd as S
from paper_2412_16434_amd import binding


def _step(dev, dtype=torch.bfloat16, d=128):
    """Two sessions of 20 and 0 cached tokens with trees of 3 and 2, of 4 / 2 heads: the calls by name, each with its arguments
    and the names of what it writes."""
    g = torch.Generator().manual_seed(5)
    rand = lambda *shape: torch.randn(shape, generator=g).to(dtype).to(dev)  # noqa: E731
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)           # noqa: E731
    fill = lambda n, dt=torch.int32: torch.full((n,), 7, dtype=dt, device=dev)  # noqa: E731
    cache = S.KVCache(rand(2, 4, 16, 2, d), rand(2, 4, 16, 2, d))
    cu, lens, parents, table = i32([0, 3, 5]), i32([20, 0]), i32([-1, 0, 0, -1, 0]), i32([[3, 1], [-1, -1]])
    q, mask = rand(5, 4, d), torch.tensor([[1], [3], [5], [1], [3]], dtype=torch.int64, device=dev)
    slots = torch.tensor([20, 21, 22, 0, 1], dtype=torch.int64, device=dev)
    return {
        "build_tables": (dict(prefix_lens=lens, new_lens=i32([3, 2]), block_table=table.clone(), free_blocks=i32([0, 2]),
                              block_size=16, n_blocks=4, total_new_tokens=5, cu_new_lens=fill(3),
                              token_offsets=fill(3, torch.int64), slot_map=fill(5, torch.int64), positions=fill(5),
                              blocks_taken=fill(1), held_blocks=i32([2, 0]), held_after=fill(2), free_begin=i32([1])),
                         ["block_table", "cu_new_lens", "token_offsets", "slot_map", "positions", "blocks_taken", "held_after"]),
        "tree_mask": (dict(parents=parents, cu_new_lens=cu, max_new_len=3, mask=torch.zeros_like(mask), prefix_lens=lens,
                           positions=fill(5)), ["mask", "positions"]),
        "tree_attn": (dict(cache=cache, layer=1, q=q, k_new=rand(5, 2, d), v_new=rand(5, 2, d), out=torch.zeros_like(q),
                           tree_mask=mask, cu_new_lens=cu, prefix_lens=lens, block_table=table, max_new_len=3,
                           max_prefix_len=20, scale=0.125), ["out"]),
        "tree_accept": (dict(draft_tokens=i32([5, 6, 7, 5, 9]), parents=parents, target_tokens=i32([7, 1, 2, 9, 4]),
                             cu_new_lens=cu, prefix_lens=lens, rows=fill(5), n_accepted=fill(2), next_tokens=fill(2),
                             new_prefix_lens=fill(2)), ["rows", "n_accepted", "next_tokens", "new_prefix_lens"]),
        "kv_commit": (dict(cache=cache, k_new=rand(2, 5, 2, d), v_new=rand(2, 5, 2, d), rows=i32([0, 2, -1, 3, 4]),
                           slot_map=slots), []),
    }


NAMES = ["build_tables", "tree_mask", "tree_attn", "tree_accept", "kv_commit"]
COMPILED = dict(zip(NAMES, ["tables", "mask", "tree", "accept", "commit"]))


class Counting:
    """The compiled module with its answers kept."""

    def __init__(self, module):
        self.module, self.answers = module, []

    def __getattr__(self, name):
        def call(*args):
            self.answers.append(getattr(self.module, name)(*args))
            return self.answers[-1]
        return call


@pytest.fixture
def counting(monkeypatch):
    calls = binding._load_draft_calls()
    assert calls, "the compiled marshalling is not built"
    counted = Counting(calls)
    monkeypatch.setattr(binding, "_draft_calls", counted)
    return counted


@pytest.mark.parametrize("name", NAMES)
def test_calls_on_the_host_are_left_to_the_general_path(name, counting):
    with pytest.raises(ValueError, match="must be a device tensor"):
        getattr(S, name)(**_step("cpu")[name][0])
    assert counting.answers == [None]
    assert getattr(counting.module, COMPILED[name])() is None
    assert all(getattr(counting.module, COMPILED[name])(*range(n)) is None for n in range(17))


@pytest.mark.parametrize("name", ["tree_attn", "kv_commit"])
def test_a_cache_that_describes_itself_takes_the_general_path(name, counting):
    class Same(S.KVCache):
        pass

    a = _step("cpu")[name][0]
    a["cache"] = Same(a["cache"].k_pool, a["cache"].v_pool)
    with pytest.raises(ValueError, match="must be a device tensor"):
        getattr(S, name)(**a)
    assert not counting.answers


def test_without_the_module_the_general_path_decides(monkeypatch):
    monkeypatch.setattr(binding, "_draft_calls", None)
    monkeypatch.setattr(binding, "_attn_call", lambda *args: None)
    for name, (a, _) in _step("cpu").items():
        with pytest.raises(ValueError, match="must be a device tensor"):
            getattr(S, name)(**a)
    assert binding._draft_calls is False, "the module is looked for again by every call"


def test_without_the_library_the_checks_come_first(monkeypatch):
    monkeypatch.setattr(binding, "_draft_calls", None)
    monkeypatch.setattr(binding, "_attn_call", None)
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding, "_LIB_PATH", "/nonexistent/libsymph.so")
    for name in ("tree_mask", "tree_accept"):
        with pytest.raises((ValueError, ImportError)):
            getattr(S, name)(**_step("cpu")[name][0])
    assert binding._draft_calls is None


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_same_call_both_ways(name, dtype, d, counting):
    results = []
    for stream in (None, torch.cuda.current_stream()):   # (a stream: the general path)
        a, written = _step("cuda:0", dtype, d)[name]
        getattr(S, name)(**a, **({} if stream is None else dict(stream=stream)))
        torch.cuda.synchronize()
        results.append([a[w] for w in written] + ([a["cache"].k_pool, a["cache"].v_pool] if "cache" in a else []))
    assert counting.answers == [0]
    for one, two in zip(*results):
        assert torch.equal(one, two)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_what_may_be_left_out(name, counting):
    a, written = _step("cuda:0")[name]
    optional = dict(build_tables=["cu_new_lens", "token_offsets", "slot_map", "positions", "blocks_taken", "held_blocks",
                                  "held_after", "free_begin"],
                    tree_mask=["prefix_lens", "positions"], tree_accept=["new_prefix_lens"])
    for k in optional.get(name, []):
        del a[k]
    getattr(S, name)(**a)
    torch.cuda.synchronize()
    assert counting.answers == [0]


BAD = [("build_tables", "slot_map", lambda t: t[:3]), ("build_tables", "cu_new_lens", lambda t: t[:2]),
       ("build_tables", "block_table", lambda t: t[:1]), ("build_tables", "new_lens", lambda t: t.long()),
       ("build_tables", "free_blocks", lambda t: t[None]), ("build_tables", "held_blocks", lambda t: t.repeat(2)[::2]),
       ("tree_mask", "mask", lambda t: t[:4]), ("tree_mask", "mask", lambda t: t[:, 0]), ("tree_mask", "positions", lambda t: t[:4]),
       ("tree_mask", "parents", lambda t: t.cpu()), ("tree_attn", "tree_mask", lambda t: t[:4]),
       ("tree_attn", "cu_new_lens", lambda t: t[:2]), ("tree_attn", "block_table", lambda t: t[:1]),
       ("tree_attn", "q", lambda t: t.float()), ("tree_attn", "k_new", lambda t: t[:, :1].contiguous()),
       ("tree_attn", "tree_mask", lambda t: t.int()), ("tree_accept", "rows", lambda t: t[:4]),
       ("tree_accept", "n_accepted", lambda t: t[:1]), ("tree_accept", "parents", lambda t: t[:4]),
       ("kv_commit", "k_new", lambda t: t[:1]), ("kv_commit", "slot_map", lambda t: t[:4]), ("kv_commit", "rows", lambda t: t.long())]


@pytest.mark.gpu
@pytest.mark.parametrize("name,argument,change", BAD, ids=[f"{n}-{a}-{i}" for i, (n, a, _) in enumerate(BAD)])
def test_what_the_general_path_refuses_it_gets(name, argument, change, counting):
    a, _ = _step("cuda:0")[name]
    a[argument] = change(a[argument])
    with pytest.raises(ValueError):
        getattr(S, name)(**a)
    assert counting.answers == [None]


@pytest.mark.gpu
def test_errors_of_the_library_are_raised(counting):
    a, _ = _step("cuda:0")["tree_attn"]
    a["layer"] = 2
    with pytest.raises(S.SymphError, match="symph_tree_attn"):
        S.tree_attn(**a)
    assert counting.answers == [-1]


@pytest.mark.gpu
def test_the_call_goes_to_the_current_stream():
    """On a side stream: a delay, the queries copied over other values, the call.  Launched anywhere else it would not wait for the
    copy and read the other values."""
    a, _ = _step("cuda:0")["tree_attn"]
    S.tree_attn(**a)
    torch.cuda.synchronize()
    want, q = a["out"].clone(), a["q"]
    a["q"] = torch.ones_like(q)
    a["out"].zero_()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        a["q"].copy_(q)
        S.tree_attn(**a)
    side.synchronize()
    assert torch.equal(want, a["out"])
