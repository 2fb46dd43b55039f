"""symph_kv_compact where calls of one launch end and calls of three begin, and symph_kv_free at the same sizes."""
import numpy as np
import pytest

import beam_ref as R
from test_gpu_kv_blocks import _compact, _free

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_blocks,entries", [(8192, 8192), (8192, 8224), (8192, 16384), (6144, 12288), (6144, 12320), (4096, 16384),
                                              (4097, 16384), (2048, 16384), (2048, 16416), (8193, 8192)])
def test_both_sides_of_the_limit(n_blocks, entries):
    rs, rows = np.random.RandomState(entries), 32
    lens, held, table, refs, _ = R.shared_pages(rs, 8, 4, 16, 40 * n_blocks // 2048 * 6, n_blocks, ahead=1)
    table = np.pad(table, ((0, 0), (0, entries // rows - table.shape[1])), constant_values=-1)
    assert table.size == entries
    for n_keep in (-1, n_blocks // 2):
        _compact(refs, n_keep, lens, held, table, 16, n_blocks // 2)
        _compact(refs, n_keep, lens, held, table, 16, 7, in_place=True)
    _free(rs.randint(0, 2, size=rows), lens, held, table, refs, 16)
