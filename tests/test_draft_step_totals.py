"""Totals that no grid takes are refused before anything is computed from them (no GPU needed)."""
import ctypes as C

import pytest

import paper_2412_16434_amd as S
from test_abi import _cache

EUNSUPPORTED = -2


@pytest.mark.parametrize("total", [3 * 2**30 * 11, 2**40, 2**50, 2**62, 2**63 - 600, 2**63 - 1])
def test_tables_of_more_tokens_than_a_grid_takes(total):
    assert S.load_library().symph_build_tables(0x10, 0x10, None, 2, 0x10, 4, 0x10, 8, None, 16, 64, total, None, None, None, None,
                                               None, None, None) == EUNSUPPORTED


def test_more_sessions_tokens_or_entries_than_a_grid_takes():
    """A grid has less than 2^32 threads along an axis."""
    lib, c = S.load_library(), _cache()
    for n in (1 << 27, 2**31 - 1):
        assert lib.symph_tree_mask(0x10, 0x10, None, n, 200, 100, 0x10, 2, None, None) == EUNSUPPORTED
        assert lib.symph_tree_accept(0x10, 0x10, 0x10, 0x10, 0x10, n, 8, 0x10, 0x10, 0x10, 0x10, None) == EUNSUPPORTED
    for n in (1 << 30, 2**31 - 1):
        assert lib.symph_kv_commit(C.byref(c), 0x10, 0x10, 4, 0x10, 0x10, n, None) == EUNSUPPORTED

    def attn(q, n, total, top):
        return lib.symph_tree_attn(C.byref(c), 0, q, 0x10, 0x10, 0x10, 0x10, 1, 0x10, 0x10, 0x10, 4, n, 32, total, top, 16, 0.1, None,
                                   0, None)
    assert attn(0x12, 1, 1 << 21, 64) == EUNSUPPORTED               # a wave per row: addresses not on 16 bytes
    assert attn(0x10, 1 << 23, 1 << 23, 1) == EUNSUPPORTED          # a tile per session
    assert lib.symph_tree_attn_workspace_bytes(C.byref(c), 1 << 23, 32, 1 << 23, 1, 16) < 0
