"""Joins of a tile's pieces at the ends of the range of values."""
import numpy as np
import pytest

import workloads as W
from test_gpu_draft_step import KINDS, Draft

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("prefix,new", [([6000], [4]), ([6000], [40]), ([5000, 5000, 2500], [6, 3, 9])])
@pytest.mark.parametrize("every", [512, 300])
def test_pieces_that_fit_and_whose_sum_does_not(dtype, d, prefix, new, every):
    """A flat softmax over values that are zero but for a few of nearly the largest size, one or none to a piece: what each piece adds
    up fits, the pieces' sum would overflow, their mean does not."""
    draft = Draft(prefix, new, dtype, d, hkv=1, g=4, seed=72)
    draft.q[...] = 0
    big = np.float32(3.0e38) if dtype == "fp32" else W.f32_to_bf16_bits(np.array([3.0e38], np.float32))[0]
    draft.v_new[...] = 0
    draft.v_pool[...] = 0
    for s, p in enumerate(prefix):
        for j in range(7, p, every):
            draft.v_pool[draft.table[s, j // draft.bs], j % draft.bs] = big
    got = draft.check()
    assert np.isfinite(got).all() and got.max() > 1e35
