"""The compiled marshalling of beam search's calls against the general path: it takes the same calls with the same results, and leaves
everything it does not take, errors above all, to the general path."""
import types

import pytest
import torch

import paper_2412_16434_amd as S
from paper_2412_16434_amd import binding


def _step(dev, dtype=torch.bfloat16):
    """Two sessions with two beams each, of 20 and 33 cached tokens in blocks of 16: the calls by name, each with its arguments and the
    names of what it writes."""
    g = torch.Generator().manual_seed(5)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)           # noqa: E731
    fill = lambda *n: torch.full(n, 7, dtype=torch.int32, device=dev)        # noqa: E731
    f32 = lambda n: torch.full((n,), 7.0, device=dev)                        # noqa: E731
    rand = lambda *shape: torch.randn(shape, generator=g).to(dtype).to(dev)  # noqa: E731
    lens, table = i32([20, 20, 33, 33]), i32([[0, 1, -1], [0, 2, -1], [3, 4, 5], [3, 6, 7]])
    refs, space = i32([2, 1, 1, 2, 1, 1, 1, 1, 0, 0]), torch.zeros(4096, dtype=torch.uint8, device=dev)
    return {
        "beam_select": (dict(logits=rand(4, 50), scores=torch.tensor([-1.0, -2.0, -1.5, -1.0], device=dev), cu_rows=i32([0, 2, 4]),
                             cu_next=i32([0, 2, 5]), max_next=3, parents=fill(5), tokens=fill(5), next_scores=f32(5), end_token=3,
                             end_scores=f32(4), workspace=space), ["parents", "tokens", "next_scores", "end_scores"]),
        "kv_fork": (dict(parents=i32([0, 0, 3, 2]), lens=lens, block_table=table, refs=refs, free_blocks=i32([8, 9]), block_size=16,
                         table_out=fill(4, 3), lens_out=fill(4), refs_after=fill(10), copy_src=fill(4), copy_dst=fill(4),
                         copy_tokens=fill(4), held_blocks=i32([0, 0, 3, 3]), held_out=fill(4), free_begin=i32([1]),
                         blocks_taken=fill(1)),
                    ["table_out", "lens_out", "refs_after", "copy_src", "copy_dst", "copy_tokens", "held_out", "blocks_taken"]),
        "kv_copy_blocks": (dict(cache=S.KVCache(rand(2, 10, 16, 2, 8), rand(2, 10, 16, 2, 8)), src_blocks=i32([1, -1, 4]),
                                dst_blocks=i32([8, 2, 9]), tokens=i32([4, 16, 20])), []),
        "kv_free": (dict(drop=i32([0, 1, 0, 0]), lens=lens, block_table=table, refs=refs, block_size=16, refs_after=fill(10),
                         free_blocks=fill(10), n_free=fill(1), held_blocks=i32([2, 2, 3, 3]), lens_after=fill(4), held_after=fill(4),
                         workspace=space, taken_blocks=i32([9, 8, 3]), taken_begin=i32([0]), taken_end=i32([1])),
                    ["refs_after", "free_blocks", "n_free", "lens_after", "held_after"]),
        "kv_compact": (dict(refs=refs, n_keep=-1, lens=lens, block_table=table, block_size=16, table_out=fill(4, 3), refs_after=fill(10),
                            block_map=fill(10), copy_src=fill(5), copy_dst=fill(5), counts=fill(3), held_blocks=i32([2, 2, 3, 3]),
                            workspace=space), ["table_out", "refs_after", "block_map", "copy_src", "copy_dst", "counts"]),
    }


NAMES = ["beam_select", "kv_fork", "kv_copy_blocks", "kv_free", "kv_compact"]
COMPILED = dict(zip(NAMES, ["select_beams", "fork_rows", "copy_blocks", "free_rows", "compact_pool"]))


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
    calls = binding._load_beam_calls()
    assert calls, "the compiled marshalling is not built"
    counted = Counting(calls)
    monkeypatch.setattr(binding, "_beam_calls", counted)
    return counted


@pytest.mark.parametrize("name", NAMES)
def test_calls_on_the_host_are_left_to_the_general_path(name, counting):
    with pytest.raises(ValueError, match="must be (a )?device tensor"):
        getattr(S, name)(**_step("cpu")[name][0])
    assert counting.answers == [None]
    assert all(getattr(counting.module, COMPILED[name])(*range(n)) is None for n in range(18))


def test_without_the_module_the_general_path_decides(monkeypatch):
    monkeypatch.setattr(binding, "_beam_calls", None)
    monkeypatch.setattr(binding, "_attn_call", lambda *args: None)
    for name, (a, _) in _step("cpu").items():
        with pytest.raises(ValueError, match="must be (a )?device tensor"):
            getattr(S, name)(**a)
    assert binding._beam_calls is False


def test_tensors_of_another_device_are_refused(monkeypatch):
    far = types.SimpleNamespace(is_cuda=True, get_device=lambda: 1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="lens is on cuda:1, the current device is cuda:0"):
        binding._on_this_device(None, held=None, lens=far)
    binding._on_this_device(5, lens=far)  # (a stream says where the call goes)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_same_call_both_ways(name, dtype, counting):
    results = []
    for stream in (None, torch.cuda.current_stream()):   # (a stream: the general path)
        a, written = _step("cuda:0", dtype)[name]
        getattr(S, name)(**a, **({} if stream is None else dict(stream=stream)))
        torch.cuda.synchronize()
        results.append([a[w] for w in written] + ([a["cache"].k_pool, a["cache"].v_pool] if "cache" in a else []))
    assert counting.answers == [0]
    for one, two in zip(*results):
        assert torch.equal(one, two)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_what_may_be_left_out(name, counting):
    optional = dict(beam_select=["end_scores", "end_token"], kv_fork=["held_blocks", "held_out", "free_begin", "blocks_taken"],
                    kv_copy_blocks=["tokens"], kv_free=["held_blocks", "lens_after", "held_after", "taken_blocks", "taken_begin", "taken_end"], kv_compact=["held_blocks"])
    a, _ = _step("cuda:0")[name]
    for k in optional[name]:
        del a[k]
    getattr(S, name)(**a)
    torch.cuda.synchronize()
    assert counting.answers == [0]


BAD = [("beam_select", "scores", lambda t: t[:3]), ("beam_select", "logits", lambda t: t.half()), ("beam_select", "logits", lambda t: t.t()),
       ("beam_select", "cu_next", lambda t: t[:2]), ("beam_select", "tokens", lambda t: t.long()),
       ("beam_select", "next_scores", lambda t: t[:4]), ("beam_select", "end_scores", lambda t: t.double()),
       ("beam_select", "workspace", lambda t: t[::2]), ("kv_fork", "table_out", lambda t: t[:3]),
       ("kv_fork", "table_out", lambda t: t[:, :2].contiguous()), ("kv_fork", "block_table", lambda t: t[:, ::2]),
       ("kv_fork", "refs_after", lambda t: t[:9]), ("kv_fork", "copy_dst", lambda t: t[:3]), ("kv_fork", "held_blocks", lambda t: t.cpu()),
       ("kv_copy_blocks", "dst_blocks", lambda t: t[:2]), ("kv_copy_blocks", "tokens", lambda t: t.long()),
       ("kv_free", "lens", lambda t: t[:3]), ("kv_free", "free_blocks", lambda t: t[:9]), ("kv_free", "drop", lambda t: t.bool()),
       ("kv_free", "block_table", lambda t: t[:3]), ("kv_compact", "block_map", lambda t: t[:9]), ("kv_compact", "counts", lambda t: t[:2]),
       ("kv_compact", "table_out", lambda t: t[:3]), ("kv_compact", "copy_dst", lambda t: t[:4])]


@pytest.mark.gpu
@pytest.mark.parametrize("name,argument,change", BAD, ids=[f"{n}-{a}-{i}" for i, (n, a, _) in enumerate(BAD)])
def test_what_the_general_path_refuses_it_gets(name, argument, change, counting):
    a, _ = _step("cuda:0")[name]
    a[argument] = change(a[argument])
    with pytest.raises(ValueError):
        getattr(S, name)(**a)
    assert counting.answers == [None]


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["beam_select", "kv_free", "kv_compact"])
def test_errors_of_the_library_are_raised(name, counting):
    a, _ = _step("cuda:0")[name]
    a["workspace"] = None
    with pytest.raises(S.SymphError, match=f"symph_{name}"):
        getattr(S, name)(**a)
    assert counting.answers == [-4]
