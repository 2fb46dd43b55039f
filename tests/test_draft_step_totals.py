"""Totals that no grid takes are refused before anything is computed from them (no GPU needed)."""
import pytest

import paper_2412_16434_amd as S

EUNSUPPORTED = -2


@pytest.mark.parametrize("total", [3 * 2**30 * 11, 2**40, 2**50, 2**62, 2**63 - 600, 2**63 - 1])
def test_tables_of_more_tokens_than_a_grid_takes(total):
    assert S.load_library().symph_build_tables(0x10, 0x10, None, 2, 0x10, 4, 0x10, 8, None, 16, 64, total, None, None, None, None,
                                               None, None, None) == EUNSUPPORTED
