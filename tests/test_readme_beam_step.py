"""README's step of beam search, run as it stands there on plain references (numpy, no GPU): counts, tables and the free list have to
agree with each other after every step, sessions that are done among them."""
import inspect
import os
import re
import textwrap
import types

import numpy as np
import pytest

import beam_ref as R
import draft_ref
import paper_2412_16434_amd as S

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")
BEAMS, STRIDE, BLOCKS, BS = 3, 12, 120, 16


def _snippet():
    text = open(README).read()
    text = text[text.index("A step of beam search"):]
    return textwrap.dedent(re.search(r"\n\n((?:    .*\n)+)", text).group(1))


class Plain:
    """The calls of the package on numpy arrays, arguments bound to the package's own signatures."""

    def __init__(self, chosen):
        self.chosen = chosen

    def __getattr__(self, name):
        def call(*args, **kw):
            bound = inspect.signature(getattr(S, name)).bind(*args, **kw)
            bound.apply_defaults()
            getattr(self, "_" + name)(types.SimpleNamespace(**bound.arguments))
        return call

    def _put(self, a, result):
        for name, value in result.items():
            if getattr(a, name, None) is not None:
                getattr(a, name)[...] = np.asarray(value).reshape(getattr(a, name).shape)

    def _beam_select(self, a):
        a.parents[...] = self.chosen

    def _kv_free(self, a):
        n, taken = len(a.drop), a.taken_blocks is not None
        self._put(a, R.free(a.drop, a.lens, a.held_blocks if a.held_blocks is not None else np.zeros(n, int), a.block_table, a.refs,
                            a.block_size, a.taken_blocks if taken else (), int(a.taken_begin[0]) if taken and a.taken_begin is not None else 0,
                            int(a.taken_end[0]) if taken else 0))

    def _kv_fork(self, a):
        begin = 0 if a.free_begin is None else int(a.free_begin[0])
        self._put(a, R.fork(a.parents, a.lens, a.held_blocks if a.held_blocks is not None else np.zeros(len(a.lens), int), a.block_table,
                            a.refs, a.free_blocks, begin, a.block_size, a.table_out))

    def _kv_copy_blocks(self, a):
        pass

    def _build_tables(self, a):
        got = draft_ref.build_tables(a.prefix_lens, a.new_lens, a.block_table, a.free_blocks, a.block_size, a.n_blocks,
                                     a.total_new_tokens, a.held_blocks, 0 if a.free_begin is None else int(a.free_begin[0]))
        a.block_table[...] = got["table"]
        self._put(a, dict(blocks_taken=got["taken"], held_after=got["held_after"], slot_map=got["slots"], cu_new_lens=got["cu"]))


def _z(*shape):
    return np.zeros(shape, np.int32)


def _counts(v, lens, held, table):
    """How many rows hold each block, by the tables."""
    counts = np.zeros(BLOCKS, int)
    for r in range(len(lens)):
        for b in table[r, :max(R.ceil_div(int(lens[r]), BS), int(held[r]))]:
            assert 0 <= b < BLOCKS, (r, v)
            counts[b] += 1
    return counts


@pytest.mark.parametrize("seed", range(5))
def test_the_step_in_the_readme(seed):
    rs, rows = np.random.RandomState(seed), 3 * BEAMS
    code = compile(_snippet(), "README.md", "exec")
    v = dict(cache=None, logits=None, scores=None, cu_rows=None, cu_next=None, width=BEAMS, tokens=None, next_scores=None, ended=None,
             space=None, n_blocks=BLOCKS, T=rows, new_lens=np.ones(rows, np.int32), lens=_z(rows), held=_z(rows),
             table=np.full((rows, STRIDE), -1, np.int32), refs=_z(BLOCKS), free=rs.permutation(BLOCKS).astype(np.int32),
             used_before=_z(1), used=_z(1), drop=_z(rows))
    # prompts of every beam, in blocks that nobody has counted yet
    prompts = rs.randint(1, 60, size=rows)
    got = draft_ref.build_tables(v["lens"], prompts, v["table"], v["free"], BS, BLOCKS, int(prompts.sum()))
    v.update(table=got["table"], held=got["held_after"], used=got["taken"], lens=prompts.astype(np.int32))
    gone = set()
    for step in range(8):
        if step in (2, 5):
            gone.add(int(rs.randint(3)))
        drop = np.array([r // BEAMS in gone for r in range(rows)])
        parents = np.arange(rows) // BEAMS * BEAMS + rs.randint(0, BEAMS, size=rows)
        v.update(drop=drop.astype(np.int32), parents=_z(rows), refs_now=_z(BLOCKS), free_now=_z(BLOCKS), n_free=_z(1), lens_now=_z(rows),
                 held_now=_z(rows), table_out=np.full((rows, STRIDE), -1, np.int32), lens_out=_z(rows), refs_out=_z(BLOCKS),
                 copy_src=_z(rows), copy_dst=_z(rows), copy_tokens=_z(rows), held_out=_z(rows), forked=_z(1), cu=_z(rows + 1),
                 slots=np.zeros(rows, np.int64), used_now=_z(1), held_next=_z(rows), new_lens=np.where(drop, 0, 1).astype(np.int32))
        before = v["lens"].copy()
        v["S"] = Plain(parents)
        exec(code, v)
        assert np.array_equal(v["lens_out"], np.where(drop, 0, before[parents]))
        # what is counted, the blocks that build_tables took behind it, and the tables are the same
        counted = v["refs_out"] + np.bincount(v["free_now"][int(v["forked"][0]):int(v["used_now"][0])], minlength=BLOCKS)
        assert np.array_equal(counted, _counts(v, v["lens_out"], v["held_next"], v["table_out"]))
        # and what is left of the list is held by nobody
        left = v["free_now"][int(v["used_now"][0]):int(v["n_free"][0])]
        assert np.all(counted[left] == 0)
        v.update(lens=v["lens_out"] + v["new_lens"], held=v["held_next"], table=v["table_out"], refs=v["refs_out"], free=v["free_now"],
                 used_before=v["forked"], used=v["used_now"])
