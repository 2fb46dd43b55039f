"""Bounds that the speculative step's attention refuses or takes, from host-side values alone (no GPU needed)."""
import ctypes as C

import paper_2412_16434_amd as S
from test_abi import _cache

EUNSUPPORTED = -2


def test_the_longest_prefixes():
    lib, c = S.load_library(), _cache()
    size = lambda *a: lib.symph_tree_attn_workspace_bytes(C.byref(c), *a)  # noqa: E731
    call = lambda far, top: lib.symph_tree_attn(C.byref(c), 0, *[0x10] * 5, 4, 0x10, 0x10, 0x10, 1 << 27, 1, 32, top, top, far, 0.1,  # noqa: E731
                                                None, 0, None)
    assert size(1, 32, 256, 256, 2**31 - 16) < 0 and call(2**31 - 16, 256) == EUNSUPPORTED
    assert size(1, 32, 4, 4, 10**9) > 0                                # one tile of rows
    assert size(4096, 32, 4096, 1, 10**6) > 0                          # many sessions: each of them is within bounds
    assert size(1, 32, 64, 64, 2**20) < 2**31


def test_sizes_that_overflow_are_refused_by_the_query():
    lib, c, top = S.load_library(), _cache(), 2**31 - 1
    size = lambda *a: lib.symph_tree_attn_workspace_bytes(C.byref(c), *a)  # noqa: E731
    for bad in ((1, 32, top, 1, 64), (1, 32, 8, top, 64), (top, 32, 8, 8, 64), (top, 32, top, top, top), (1, 8 * (top // 8), 8, 8, 64)):
        assert size(*bad) < 0, bad
