"""The example of a drafted step: trees give the tokens that one token a step gives, in fewer steps."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import drafted_steps as E  # noqa: E402


def test_drafts_are_trees_over_the_history():
    tokens, parents = E.draft_from_history([1, 2, 3, 4, 1, 2, 3, 5, 1, 2], branches=4, depth=3)
    assert tokens == [2, 3, 5, 1, 4, 1] and parents == [-1, 0, 1, 2, 1, 4]   # 3 5 1 and 3 4 1 share their first node
    assert E.draft_from_history([7, 8, 9], 4, 3) == ([9], [-1])
    assert E.draft_from_history([7, 7], 0, 3) == ([7], [-1])
    assert all(p < i for i, p in enumerate(parents))


@pytest.mark.gpu
@pytest.mark.parametrize("block_size,sessions", [(16, 3), (5, 1), (1, 2)])
def test_trees_give_the_same_tokens_in_fewer_steps(block_size, sessions):
    model = E.Model(layers=2)
    g = torch.Generator().manual_seed(sessions)
    # (prompts that repeat themselves: there is something to draft from the first step on)
    prompts = [(torch.randint(0, 512, (9 + s,), generator=g).tolist() * 3) for s in range(sessions)]
    one, steps_one = E.generate(model, prompts, 48, branches=0, block_size=block_size)
    many, steps_many = E.generate(model, prompts, 48, block_size=block_size)
    assert one == many and steps_one == 47 and steps_many < steps_one


@pytest.mark.gpu
def test_the_script_runs(capsys):
    assert E.main(["--sessions", "2", "--tokens", "40"]) == 0
    assert "2 of 2 sessions have the same tokens both ways" in capsys.readouterr().out
    assert E.main(["--sessions", "2", "--tokens", "20", "--dtype", "bf16"]) == 0
