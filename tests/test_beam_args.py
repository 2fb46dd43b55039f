"""What the entry points of beam search refuse, before anything touches a GPU (these run without one)."""
import ctypes as C

import numpy as np
import pytest
import torch

import beam_ref as R
import paper_2412_16434_amd as S
from test_abi import _cache

EINVAL, EUNSUPPORTED, EWORKSPACE = -1, -2, -4
BIG = 1 << 40


def test_beam_select_refuses():
    lib = S.load_library()

    def call(logits=0x10, stride=100, dtype=0, rows=4, vocab=100, scores=0x20, cu=0x30, cu_next=0x40, n=2, total=8, most=4, end=3,
             parents=0x50, tokens=0x60, best=0x70, ends=None, ws=0x100, ws_bytes=BIG):
        return lib.symph_beam_select(logits, stride, dtype, rows, vocab, scores, cu, cu_next, n, total, most, end, parents, tokens, best,
                                     ends, ws, ws_bytes, None)
    for bad in (dict(logits=None), dict(stride=99), dict(rows=-1), dict(vocab=0), dict(vocab=-1), dict(scores=None), dict(cu=None),
                dict(cu_next=None), dict(n=-1), dict(total=-1), dict(most=-1), dict(end=100), dict(parents=None), dict(tokens=None),
                dict(best=None), dict(best=0x20), dict(ws_bytes=-1)):
        assert call(**bad) == EINVAL, bad
    assert call(dtype=2) == EUNSUPPORTED and call(most=65) == EUNSUPPORTED and call(rows=1 << 30) == EUNSUPPORTED
    assert call(n=1 << 30) == EUNSUPPORTED
    assert call(ws=None) == EWORKSPACE and call(ws_bytes=8) == EWORKSPACE
    assert call(n=0) == 0


def test_fork_refuses():
    lib = S.load_library()

    def call(parents=0x10, out=4, lens=0x20, held=None, rows=4, table=0x30, stride=8, bs=16, blocks=64, refs=0x40, free=0x50, n_free=8,
             begin=None, table_out=0x60, lens_out=0x70, held_out=None, after=0x80, src=0x90, dst=0xA0, tokens=0xB0, taken=None):
        return lib.symph_kv_fork(parents, out, lens, held, rows, table, stride, bs, blocks, refs, free, n_free, begin, table_out, lens_out,
                                 held_out, after, src, dst, tokens, taken, None)
    for bad in (dict(parents=None), dict(out=-1), dict(lens=None), dict(rows=-1), dict(table=None), dict(stride=-1), dict(bs=0),
                dict(blocks=0), dict(refs=None), dict(free=None), dict(n_free=-1), dict(table_out=None), dict(lens_out=None),
                dict(after=None), dict(src=None), dict(dst=None), dict(tokens=None), dict(after=0x40), dict(table_out=0x30),
                dict(lens_out=0x20), dict(held=0x21, held_out=0x21), dict(begin=0x51, taken=0x51)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=8193) == EUNSUPPORTED and call(out=8193) == EUNSUPPORTED


def test_copy_blocks_refuses():
    lib = S.load_library()

    def call(cache=None, src=0x10, dst=0x20, tokens=None, n=4):
        c = _cache() if cache is None else cache
        return lib.symph_kv_copy_blocks(C.byref(c), src, dst, tokens, n, None)
    for bad in (dict(src=None), dict(dst=None), dict(n=-1), dict(cache=_cache(n_layers=0)), dict(cache=_cache(block_stride=8))):
        assert call(**bad) == EINVAL, bad
    assert lib.symph_kv_copy_blocks(None, 0x10, 0x20, None, 4, None) == EINVAL
    assert call(cache=_cache(dtype=9)) == EUNSUPPORTED and call(cache=_cache(k_base=0x1002)) == EUNSUPPORTED
    assert call(cache=_cache(n_layers=65536)) == EUNSUPPORTED
    assert call(n=0) == 0


def test_free_refuses():
    lib = S.load_library()

    def call(drop=0x10, lens=0x20, held=None, rows=4, table=0x30, stride=8, bs=16, blocks=64, refs=0x40, after=0x50, free=0x60, n_free=0x70,
             taken=None, n_taken=0, taken_end=None, ws=0x100, ws_bytes=BIG):
        return lib.symph_kv_free(drop, lens, held, rows, table, stride, bs, blocks, refs, after, free, n_free, None, None, taken, n_taken,
                                 None, taken_end, ws, ws_bytes, None)
    for bad in (dict(drop=None), dict(lens=None), dict(rows=-1), dict(table=None), dict(stride=-1), dict(bs=0), dict(blocks=0),
                dict(refs=None), dict(after=None), dict(free=None), dict(n_free=None), dict(after=0x40), dict(free=0x40), dict(free=0x50),
                dict(ws_bytes=-1), dict(n_taken=-1), dict(taken=0x80, n_taken=4), dict(taken=0x60, n_taken=4, taken_end=0x90)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=1 << 30) == EUNSUPPORTED
    assert call(ws=None) == EWORKSPACE and call(ws_bytes=3) == EWORKSPACE


def test_compact_refuses():
    lib = S.load_library()

    def call(refs=0x10, blocks=64, keep=-1, lens=0x20, held=None, rows=4, table=0x30, stride=8, bs=16, table_out=0x40, after=0x50,
             where=0x60, src=0x70, dst=0x80, pairs=32, counts=0x90, ws=0x100, ws_bytes=BIG):
        return lib.symph_kv_compact(refs, blocks, keep, lens, held, rows, table, stride, bs, table_out, after, where, src, dst, pairs,
                                    counts, ws, ws_bytes, None)
    for bad in (dict(refs=None), dict(blocks=0), dict(lens=None), dict(rows=-1), dict(table=None), dict(stride=-1), dict(bs=0),
                dict(table_out=None), dict(after=None), dict(where=None), dict(src=None), dict(dst=None), dict(dst=0x70), dict(pairs=-1),
                dict(counts=None), dict(after=0x10), dict(where=0x10), dict(where=0x50), dict(ws_bytes=-1)):
        assert call(**bad) == EINVAL, bad
    assert call(rows=1 << 30) == EUNSUPPORTED
    assert call(ws=None) == EWORKSPACE and call(ws_bytes=3) == EWORKSPACE


def test_workspace_queries():
    lib = S.load_library()
    assert lib.symph_beam_select_workspace_bytes(8, 1000, 4) > 0 and lib.symph_beam_select_workspace_bytes(0, 1000, 4) == 0
    for bad in ((-1, 1000, 4), (8, 0, 4), (8, 1000, -1), (8, 1000, 65)):
        assert lib.symph_beam_select_workspace_bytes(*bad) < 0, bad
    for query in (lib.symph_kv_free_workspace_bytes, lib.symph_kv_compact_workspace_bytes):
        assert query(1) > 0 and query(2 ** 31 - 1) > 0 and query(0) < 0 and query(-1) < 0
    with pytest.raises(S.SymphError):
        S.kv_free_workspace_bytes(0)
    with pytest.raises(S.SymphError):
        S.beam_select_workspace_bytes(1, 1, 65)


def test_the_binding_checks_tensors():
    i32, f32 = torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    table = torch.zeros((4, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="n_rows"):
        S.beam_select(torch.zeros(8), f32, i32, i32, 1, i32, i32, f32)
    with pytest.raises(ValueError, match="n_rows"):
        S.beam_select(torch.zeros((4, 8), dtype=torch.float16), f32, i32, i32, 1, i32, i32, f32)
    with pytest.raises(ValueError, match="device"):
        S.beam_select(torch.zeros((4, 8)), f32, i32, i32, 1, i32, i32, f32)
    with pytest.raises(ValueError, match="device"):
        S.kv_fork(i32, i32, table, i32, i32, 16, table, i32, i32, i32, i32, i32)
    with pytest.raises(ValueError, match="table_out|device"):
        S.kv_fork(i32, i32, table, i32, i32, 16, table[:, :1], i32, i32, i32, i32, i32)
    with pytest.raises(ValueError, match="block_table"):
        S.kv_fork(i32, i32, None, i32, i32, 16, table, i32, i32, i32, i32, i32)
    pool = torch.zeros((2, 8, 16, 1, 64))
    with pytest.raises(ValueError, match="device"):
        S.kv_copy_blocks(S.KVCache(pool, pool), i32, i32)
    with pytest.raises(ValueError, match="device"):
        S.kv_free(None, None, None, i32, 16, i32, i32, i32)
    with pytest.raises(ValueError, match="block_table"):
        S.kv_free(i32, i32, None, i32, 16, i32, i32, i32)
    with pytest.raises(ValueError, match="device"):
        S.kv_compact(i32, -1, i32, table, 16, table, i32, i32, i32, i32, i32)


def test_the_references_against_worked_examples():
    x = np.log(np.array([[0.5, 0.3, 0.2], [0.1, 0.1, 0.8]]))
    got = R.beam_select(x, np.zeros(2), [0, 2], [0, 3], 3, 0)
    assert got["parents"].tolist() == [1, 0, 0] and got["tokens"].tolist() == [2, 1, 2]
    assert np.allclose(got["end_scores"], [np.log(0.5), -np.inf])
    table, refs = np.array([[3, 1], [3, 2]]), np.array([0, 1, 1, 2, 0])
    got = R.fork([1, 1, -1], [6, 7], [0, 0], table, refs, [4, 0], 0, 4, np.full((3, 2), -1))
    assert got["table_out"].tolist() == [[3, 2], [3, 4], [-1, -1]] and got["refs_after"].tolist() == [0, 0, 1, 2, 1]
    assert got["copy_src"] == [-1, 2, -1] and got["copy_dst"] == [-1, 4, -1] and got["copy_tokens"] == [0, 3, 0]
    got = R.free([0, 1], [6, 7], [0, 0], table, refs, 4)
    assert got["refs_after"].tolist() == [0, 1, 0, 1, 0] and got["free_blocks"].tolist() == [0, 2, 4, -1, -1] and got["n_free"] == [3]
    got = R.compact(refs, -1, [6, 7], [0, 0], table, 4, 2, table)
    assert got["table_out"].tolist() == [[0, 1], [0, 2]] and got["refs_after"].tolist() == [2, 1, 1, 0, 0]
    assert got["copy_src"] == [3, -1] and got["copy_dst"] == [0, -1] and got["counts"] == [3, 1, 0]
