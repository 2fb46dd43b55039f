"""What the speculative step's entry points refuse, before anything touches a GPU (these run without one)."""
import ctypes as C

import numpy as np
import pytest
import torch

import draft_ref as R
import paper_2412_16434_amd as S
from test_abi import _cache

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -4


def test_build_tables_refuses():
    lib = S.load_library()

    def call(prefix=0x10, new=0x10, held=None, n=2, table=0x10, stride=4, free=0x10, n_free=8, begin=None, bs=16, blocks=64,
             total=10, cu=0x10, taken=None, after=None):
        return lib.symph_build_tables(prefix, new, held, n, table, stride, free, n_free, begin, bs, blocks, total, cu, None, None,
                                      None, taken, after, None)
    for bad in (dict(prefix=None), dict(new=None), dict(n=-1), dict(table=None), dict(stride=0), dict(stride=-1), dict(free=None),
                dict(n_free=-1), dict(bs=0), dict(blocks=0), dict(total=-1), dict(total=1 << 31), dict(held=0x20, after=0x20),
                dict(begin=0x30, taken=0x30)):
        assert call(**bad) == EINVAL, bad


def test_tree_mask_refuses():
    lib = S.load_library()

    def call(parents=0x10, cu=0x10, n=2, total=200, top=100, mask=0x10, words=2):
        return lib.symph_tree_mask(parents, cu, None, n, total, top, mask, words, None, None)
    for bad in (dict(parents=None), dict(cu=None), dict(n=-1), dict(total=-1), dict(total=99), dict(top=-1), dict(mask=None),
                dict(words=1), dict(words=-1)):
        assert call(**bad) == EINVAL, bad
    assert call(total=5000, top=4097, words=65) == EUNSUPPORTED
    assert call(n=0) == 0 and call(top=0) == 0


def test_tree_attn_refuses():
    lib = S.load_library()

    def call(cache=None, layer=0, q=0x10, mask=0x10, words=1, cu=0x10, lens=0x10, table=0x10, stride=4, n=1, hq=32, total=4, top=4,
             far=16, scale=0.1, ws=None, ws_bytes=0):
        c = _cache() if cache is None else cache
        return lib.symph_tree_attn(C.byref(c), layer, q, 0x10, 0x10, 0x10, mask, words, cu, lens, table, stride, n, hq, total, top,
                                   far, scale, ws, ws_bytes, None)
    for bad in (dict(layer=2), dict(layer=-1), dict(q=None), dict(mask=None), dict(words=0), dict(words=-1), dict(cu=None),
                dict(lens=None), dict(table=None), dict(stride=0), dict(stride=-1), dict(n=-1), dict(hq=12), dict(hq=0),
                dict(total=-1), dict(top=5), dict(top=-1), dict(far=-1), dict(far=65), dict(total=100, top=65), dict(scale=0.0),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(ws_bytes=-1), dict(cache=_cache(block_stride=8)),
                dict(cache=_cache(n_blocks=0))):
        assert call(**bad) == EINVAL, bad
    assert lib.symph_tree_attn(None, 0, *[0x10] * 5, 1, 0x10, 0x10, 0x10, 4, 1, 32, 4, 4, 16, 0.1, None, 0, None) == EINVAL
    assert call(cache=_cache(head_dim=80, block_stride=16 * 8 * 80)) == EUNSUPPORTED
    assert call(cache=_cache(dtype=3)) == EUNSUPPORTED
    assert call(total=1 << 30, n=1) == EUNSUPPORTED
    assert call(far=50000, stride=4000) == EWORKSPACE
    assert call(n=0) == 0 and call(total=0, top=0) == 0


def test_tree_attn_workspace_query():
    lib, c = S.load_library(), _cache()
    size = lambda *a, cache=c: lib.symph_tree_attn_workspace_bytes(C.byref(cache), *a)  # noqa: E731
    assert size(1, 32, 8, 8, 64) == 0                        # a short prefix is not cut
    assert size(1, 32, 8, 8, 50000) > 0
    for bad in ((-1, 32, 8, 8, 64), (1, 0, 8, 8, 64), (1, 12, 8, 8, 64), (1, 32, -1, 8, 64), (1, 32, 8, -1, 64), (1, 32, 8, 8, -1)):
        assert size(*bad) < 0, bad
    assert lib.symph_tree_attn_workspace_bytes(None, 1, 32, 8, 8, 64) < 0
    assert size(1, 32, 8, 8, 64, cache=_cache(n_kv_heads=0)) < 0


def test_tree_accept_and_commit_refuse():
    lib = S.load_library()

    def accept(draft=0x10, parents=0x10, target=0x10, cu=0x10, lens=0x10, n=2, total=8, rows=0x10, counts=0x10, nxt=0x10, after=0x10):
        return lib.symph_tree_accept(draft, parents, target, cu, lens, n, total, rows, counts, nxt, after, None)
    for bad in (dict(draft=None), dict(parents=None), dict(target=None), dict(cu=None), dict(lens=None), dict(n=-1), dict(total=-1),
                dict(rows=None), dict(counts=None), dict(nxt=None)):
        assert accept(**bad) == EINVAL, bad
    assert accept(n=0) == 0

    def commit(cache=None, k=0x10, v=0x10, n_rows=4, rows=0x10, slots=0x10, n=4):
        c = _cache() if cache is None else cache
        return lib.symph_kv_commit(C.byref(c), k, v, n_rows, rows, slots, n, None)
    for bad in (dict(k=None), dict(v=None), dict(n_rows=-1), dict(rows=None), dict(slots=None), dict(n=-1),
                dict(cache=_cache(n_layers=0))):
        assert commit(**bad) == EINVAL, bad
    assert lib.symph_kv_commit(None, 0x10, 0x10, 4, 0x10, 0x10, 4, None) == EINVAL
    assert commit(k=0x12) == EUNSUPPORTED and commit(cache=_cache(dtype=9)) == EUNSUPPORTED
    assert commit(n=0) == 0 and commit(n_rows=0) == 0


def test_the_binding_checks_tensors():
    i32 = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        S.tree_mask(i32, i32, 1, torch.zeros((4, 1), dtype=torch.int64))
    with pytest.raises(ValueError, match="mask"):
        S.tree_mask(i32, i32, 1, torch.zeros((3, 1), dtype=torch.int64))
    with pytest.raises(ValueError, match="device"):
        S.tree_accept(i32, i32, i32, i32, i32, i32, i32, i32)
    with pytest.raises(ValueError, match="device"):
        S.build_tables(i32, i32, torch.zeros((4, 2), dtype=torch.int32), i32, 16, 8, 4)
    with pytest.raises(ValueError, match="2-D"):
        S.build_tables(i32, i32, i32, i32, 16, 8, 4)
    pool = torch.zeros((2, 8, 16, 1, 64))
    with pytest.raises(ValueError, match="n_rows"):
        S.kv_commit(S.KVCache(pool, pool), torch.zeros((2, 5, 1, 32)), torch.zeros((2, 5, 1, 32)), i32, i32)


def test_reference_masks_and_paths():
    """The references against worked examples."""
    sees = R.ancestors(np.array([-1, 0, 0, 1, 9, 4]))
    assert [np.flatnonzero(r).tolist() for r in sees] == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5]]
    assert R.pack_bits([sees], 1).ravel().tolist() == [1, 3, 5, 11, 16, 48]
    assert R.accept([7, 5, 5, 6, 6], [-1, 0, 0, 1, 2], [5, 6, 6, 9, 9]) == [0, 1, 3]
    assert R.accept([7, 4, 5], [-1, 0, 0], [5, 0, 0]) == [0, 2] and R.accept([], [], []) == []
    got = R.build_tables(np.array([3, 4]), np.array([2, 1]), np.array([[8, -1], [9, -1]]), np.array([5, 6]), 4, 10, 3)
    assert got["table"].tolist() == [[8, 5], [9, 6]] and got["slots"].tolist() == [35, 20, 24] and got["taken"].tolist() == [2]
