"""Steps of beam search in which sessions end: their rows dropped, their blocks listed, taken by forks and by new tokens of the same step."""
import numpy as np
import pytest
import torch

import beam_ref as R
import paper_2412_16434_amd as S

DEV = "cuda:0"


def test_a_dropped_row_is_forked_with_its_new_length():
    """On the references: the lengths from before would give a dropped row's blocks back twice."""
    table, refs = np.array([[3, 1], [3, 2]], np.int32), np.array([0, 1, 1, 2, 0], np.int32)
    lens, held = np.array([6, 7]), np.array([2, 2])
    freed = R.free([0, 1], lens, held, table, refs, 4)
    out = np.full((2, 2), -1)
    right = R.fork([0, 0], freed["lens_after"], freed["held_after"], table, freed["refs_after"], freed["free_blocks"], 0, 4, out)
    assert right["refs_after"].tolist() == [1, 1, 0, 2, 0] and right["table_out"].tolist() == [[3, 1], [3, 0]]
    twice = R.fork([0, 0], lens, held, table, freed["refs_after"], freed["free_blocks"], 0, 4, out)
    assert twice["refs_after"].min() == -1


class Sessions:
    """Rows of a paged cache and, on the host, the tokens that each has to hold (every token's K,V hold its number)."""

    def __init__(self, rows, bs, n_blocks, stride, layers=2):
        self.bs, self.n_blocks, self.stride, self.rows = bs, n_blocks, stride, rows
        pool = lambda: torch.zeros((layers, n_blocks, bs, 1, 64), device=DEV)  # noqa: E731
        self.cache = S.KVCache(pool(), pool())
        self.space = torch.empty(S.kv_free_workspace_bytes(n_blocks), dtype=torch.uint8, device=DEV)
        self.lens, self.held, self.table = self.z(rows), self.z(rows), self.z(rows, stride) - 1
        self.refs, self.begin, self.used = self.z(n_blocks), self.z(1), self.z(1)
        order = np.random.RandomState(0).permutation(n_blocks)
        self.free = torch.from_numpy(order.astype(np.int32)).to(DEV)
        self.tokens, self.next = [[] for _ in range(rows)], 1

    @staticmethod
    def z(*shape):
        return torch.zeros(shape, dtype=torch.int32, device=DEV)

    def append(self, new):
        """``new[r]`` tokens more for every row, from entry ``used`` of the list on."""
        total, n = int(sum(new)), self.rows
        cu, slots, held, used = self.z(n + 1), torch.full((total,), -1, dtype=torch.int64, device=DEV), self.z(n), self.z(1)
        new_lens = torch.tensor([int(x) for x in new], dtype=torch.int32).to(DEV)
        S.build_tables(self.lens, new_lens, self.table, self.free, self.bs, self.n_blocks, total, cu_new_lens=cu, slot_map=slots,
                       blocks_taken=used, held_blocks=self.held, held_after=held, free_begin=self.begin)
        made = np.arange(self.next, self.next + total)
        self.next += total
        layers, _, _, hkv, d = self.cache.k_pool.shape
        k = torch.from_numpy(made.astype(np.float32)).to(DEV)[None, :, None, None].expand(layers, total, hkv, d).contiguous()
        S.kv_commit(self.cache, k, -k, torch.arange(total, dtype=torch.int32, device=DEV), slots)
        self.lens, self.held, self.used, at = self.lens + new_lens, held, used, 0
        for r in range(n):
            self.tokens[r] = self.tokens[r] + made[at:at + int(new[r])].tolist()
            at += int(new[r])

    def step(self, drop, parents):
        n, b = len(parents), self.n_blocks
        refs, free, n_free, lens, held = self.z(b), self.z(b), self.z(1), self.z(self.rows), self.z(self.rows)
        S.kv_free(torch.tensor(drop, dtype=torch.int32).to(DEV), self.lens, self.table, self.refs, self.bs, refs, free, n_free,
                  held_blocks=self.held, lens_after=lens, held_after=held, workspace=self.space, taken_blocks=self.free,
                  taken_begin=self.begin, taken_end=self.used)
        out, after, held_out, used = self.z(n, self.stride) - 1, self.z(b), self.z(n), self.z(1)
        lens_out, src, dst, count = self.z(n), self.z(n), self.z(n), self.z(n)
        S.kv_fork(torch.tensor(parents, dtype=torch.int32).to(DEV), lens, self.table, refs, free, self.bs, out, lens_out, after, src, dst, count,
                  held_blocks=held, held_out=held_out, blocks_taken=used)
        S.kv_copy_blocks(self.cache, src, dst, count)
        self.tokens = [[] if not 0 <= p < self.rows or drop[p] else list(self.tokens[p]) for p in parents]
        self.rows, self.table, self.lens, self.held, self.refs, self.free, self.begin, self.used = (
            n, out, lens_out, held_out, after, free, used, used.clone())

    def check(self):
        torch.cuda.synchronize()
        lens, held, table = (t.cpu().numpy() for t in (self.lens, self.held, self.table))
        assert lens.tolist() == [len(t) for t in self.tokens]
        counts = np.zeros(self.n_blocks, int)
        k, v = self.cache.k_pool[:, :, :, 0, ::63].cpu().numpy(), self.cache.v_pool[:, :, :, 0, ::63].cpu().numpy()
        for r, tokens in enumerate(self.tokens):
            assert np.all(table[r, held[r]:] == -1)
            counts[table[r, :held[r]]] += 1
            at = np.arange(len(tokens))
            blocks, want = table[r, at // self.bs], np.array(tokens, np.float32)[None, :, None]
            assert np.array_equal(k[:, blocks, at % self.bs], np.broadcast_to(want, (k.shape[0], len(tokens), 2))), r
            assert np.array_equal(v[:, blocks, at % self.bs], np.broadcast_to(-want, (k.shape[0], len(tokens), 2))), r
        # what is counted, and the blocks taken behind it
        begin, used, free = int(self.begin[0]), int(self.used[0]), self.free.cpu().numpy()
        taken = np.bincount(free[begin:used], minlength=self.n_blocks)
        assert np.array_equal(self.refs.cpu().numpy() + taken, counts)
        left = free[used:]
        assert np.all(counts[left[left >= 0]] == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("sessions,beams,bs,n_blocks,stride", [(4, 3, 4, 200, 14), (3, 5, 1, 900, 40), (40, 8, 16, 9000, 60), (7, 4, 16, 400, 12)])
def test_steps_with_sessions_that_end(sessions, beams, bs, n_blocks, stride):
    rs = np.random.RandomState(sessions)
    rows = sessions * beams
    state = Sessions(rows, bs, n_blocks, stride)
    state.append(rs.randint(1, stride * bs // 2, size=rows))
    state.check()
    gone = np.zeros(sessions, bool)
    for step in range(8):
        if step in (1, 2, 5):
            gone[rs.randint(sessions)] = True
        of_row = np.arange(rows) // beams
        drop = gone[of_row].astype(int).tolist()
        parents = of_row * beams + rs.randint(0, beams, size=rows)
        parents = np.where(gone[of_row] & (rs.random_sample(rows) < 0.5), -1, parents).tolist()   # (a dropped row as parent: an empty row)
        state.step(drop, parents)
        state.check()
        state.append(np.where(gone[of_row], 0, 1))
        state.check()


@pytest.mark.gpu
def test_rows_of_ended_sessions_go_to_new_ones():
    """A dropped session's rows begin again as another session's: its prompt takes blocks that were listed in the same step."""
    state = Sessions(6, 4, 80, 10)
    state.append([9, 13, 7, 22, 5, 18])
    for step in range(6):
        drop = [int(r // 2 == step % 3) for r in range(6)]
        state.step(drop, [1, 0, 3, 3, 4, 5])
        state.check()
        state.append([17 if d else 1 for d in drop])
        state.check()
