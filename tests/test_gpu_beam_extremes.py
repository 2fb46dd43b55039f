"""symph_beam_select where a wave carries a value at an end of its type from tile to tile: forced tokens, masked rows, rows that end in a
part of a tile."""
import numpy as np
import pytest
import torch

from test_gpu_beam_select import BF16, DEV, FP32, INF, _call, _check, _scores, _starts

pytestmark = pytest.mark.gpu
TILE = 2048
KINDS = 6


def _rows(rows, first_tiles, tiles, dtype, seed):
    """Rows of `tiles` tiles and 37 values more, in turn: a large value and nothing else, a large value in a row without a mask, one in the
    last whole tile, one among NaN, an ordinary row of few tokens, two of the same.  Large values are in the first tiles (one to a
    wave), of every magnitude."""
    rs, vocab = np.random.RandomState(seed), tiles * TILE + 37
    large = [INF, torch.finfo(dtype).max, 1e30, 1e13, 1e10, 4e9, -1e10, -1e30, torch.finfo(dtype).min]
    logits = torch.full((rows, vocab), -INF)
    end = 11
    for r in range(rows):
        kind, v, at = r % KINDS, large[r // KINDS % len(large)], int(rs.randint(first_tiles * TILE))
        if kind == 0:
            at = end
        if kind == 1:
            logits[r] = torch.from_numpy(rs.standard_normal(vocab).astype(np.float32))
        if kind == 2:
            at += (tiles - first_tiles) * TILE
        if kind == 3:
            logits[r] = float("nan")
        if kind == 4:
            few = rs.randint(vocab, size=40)
            logits[r, few] = torch.from_numpy(rs.standard_normal(40).astype(np.float32))
        else:
            logits[r, at] = v
        if kind == 5:
            logits[r, at + first_tiles * TILE] = v
    return logits.to(dtype).to(DEV), end


# (rows, tiles in front of a wave's second one, whole tiles: eight, four, two and one waves to a part, and several parts)
SHAPES = [(516, 8, 17), (822, 4, 9), (1368, 2, 5), (2052, 1, 3), (72, 8, 62)]


@pytest.mark.parametrize("rows,first_tiles,tiles", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_large_values_that_are_carried_over_tiles(rows, first_tiles, tiles, dtype):
    logits, end = _rows(rows, first_tiles, tiles, dtype, rows)
    _check(logits, _scores(rows, 2), [1] * rows, [5] * rows, end=end)
    _check(logits, _scores(rows, 3), [KINDS] * (rows // KINDS), [9] * (rows // KINDS), end=end)


@pytest.mark.parametrize("rows,first_tiles,tiles", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("value", [INF, 1e30, 1e10])
def test_a_forced_token_is_certain(rows, first_tiles, tiles, dtype, value):
    """One token of a row is possible: its probability is 1, and the score stays what it was."""
    vocab, scores = tiles * TILE + 37, _scores(rows, 4)
    at = np.random.RandomState(rows).randint(vocab, size=rows)
    logits = torch.full((rows, vocab), -INF, dtype=dtype, device=DEV)
    logits[torch.arange(rows), torch.from_numpy(at)] = value
    got = _call(logits, scores, _starts([1] * rows), _starts([2] * rows), 2, -1, behind=0)
    assert np.array_equal(got["tokens"][::2], at) and np.array_equal(got["parents"][::2], np.arange(rows))
    assert np.array_equal(got["next_scores"][::2], scores)
    assert np.all(got["tokens"][1::2] == -1) and np.all(got["next_scores"][1::2] == -INF)
