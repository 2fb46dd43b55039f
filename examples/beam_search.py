"""Beam search over the paged cache: the operators of a step, run together by a small model with random weights.

    python examples/beam_search.py [--sessions 3] [--beams 4] [--tokens 24] [--dtype bf16]

Every session keeps its best continuations.  A beam is a row of the block table; beams of a session share the blocks of what they
have in common.  A step, behind the model's logits for every beam's last token:

    beam_select      the best continuations of every session, and which beam each continues
    kv_free          blocks taken since the last step are counted, a new free list
    kv_fork          a table row for each continuation: full blocks shared, what to copy of blocks that are still being filled
    kv_copy_blocks   those copies, all layers
    build_tables     a place for every beam's next token, whose K,V rows kv_commit then writes

Every few steps the pool is packed together (kv_compact, kv_copy_blocks), as a server does that has to give the end of its pool
back.  Continuations that end compete by score per token.  The script runs the same search without a cache as well (every beam's whole
sequence through the model again) and compares: the sequences have to be the same (in bf16 a near tie may fall the other way).
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import paper_2412_16434_amd as S  # noqa: E402
from drafted_steps import DEV, Model  # noqa: E402


class Scorer(Model):
    """The drafted steps' model, asked for logits."""

    def logits(self, tokens, positions, attend, rows):
        """Logits of ``rows`` and the K,V rows of all layers; ``attend(layer, q, k, v)`` is the attention."""
        x, t = self.embed[tokens.long()], tokens.shape[0]
        k_new = torch.empty((self.layers, t, self.hkv, self.d), dtype=self.dtype, device=DEV)
        v_new = torch.empty_like(k_new)
        for i in range(self.layers):
            h = self.norm(x)
            q = self.rotate((h @ self.wq[i]).view(t, self.hq, self.d), positions)
            k_new[i] = self.rotate((h @ self.wk[i]).view(t, self.hkv, self.d), positions)
            v_new[i] = (h @ self.wv[i]).view(t, self.hkv, self.d)
            x = x + attend(i, q, k_new[i], v_new[i]).reshape(t, -1) @ self.wo[i]
            h = self.norm(x)
            x = x + (torch.nn.functional.silu(h @ self.gate[i]) * (h @ self.up[i])) @ self.down[i]
        return (self.norm(x[rows]).float() @ self.embed.float().T) / 8, k_new, v_new


def i32(values):
    return torch.tensor(values, dtype=torch.int32).to(DEV)


class Pages:
    """The paged cache of some sessions' beams: tables, lengths, counts and the free list, and what a step does to them."""

    def __init__(self, model, n_rows, max_tokens, block_size):
        self.model, self.bs, self.stride = model, block_size, -(-max_tokens // block_size) + 1
        self.n_blocks = n_rows * self.stride * 2
        pool = lambda: torch.zeros((model.layers, self.n_blocks, block_size, model.hkv, model.d), dtype=model.dtype,  # noqa: E731
                                   device=DEV)
        self.cache = S.KVCache(pool(), pool())
        self.refs = self.zeros(self.n_blocks)
        self.space = torch.empty(max(S.kv_free_workspace_bytes(self.n_blocks), S.kv_compact_workspace_bytes(self.n_blocks)),
                                 dtype=torch.uint8, device=DEV)
        self.free, self.n_free, self.used = self.zeros(self.n_blocks), self.zeros(1), self.zeros(1)
        self.lens = self.held = self.table = None
        self.count()

    @staticmethod
    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.int32, device=DEV)

    def rows(self, n):
        """``n`` rows without a token."""
        self.lens, self.held, self.table = self.zeros(n), self.zeros(n), self.zeros(n, self.stride).fill_(-1)

    def places(self, new_lens):
        """Blocks for the rows' new tokens: (offsets, slot map)."""
        total, n = sum(new_lens), len(new_lens)
        cu, slots, held = self.zeros(n + 1), torch.empty(total, dtype=torch.int64, device=DEV), self.zeros(n)
        self.begin, self.used = self.used, self.zeros(1)
        S.build_tables(self.lens, i32(new_lens), self.table, self.free, self.bs, self.n_blocks, total, cu_new_lens=cu, slot_map=slots,
                       blocks_taken=self.used, held_blocks=self.held, held_after=held, free_begin=self.begin)
        self.held = held
        return cu, slots

    def count(self, taken=False):
        """The counts with the blocks that ``places`` took, and a new free list."""
        refs, free = self.zeros(self.n_blocks), self.zeros(self.n_blocks)
        S.kv_free(None, None, None, self.refs, self.bs, refs, free, self.n_free, workspace=self.space,
                  **(dict(taken_blocks=self.free, taken_begin=self.begin, taken_end=self.used) if taken else {}))
        self.refs, self.free, self.used = refs, free, self.zeros(1)

    def fork(self, parents):
        """Rows that continue rows ``parents``."""
        n = parents.shape[0]
        table, lens, held, refs, used = self.zeros(n, self.stride), self.zeros(n), self.zeros(n), self.zeros(self.n_blocks), self.zeros(1)
        src, dst, tokens = self.zeros(n), self.zeros(n), self.zeros(n)
        S.kv_fork(parents, self.lens, self.table, self.refs, self.free, self.bs, table, lens, refs, src, dst, tokens,
                  held_blocks=self.held, held_out=held, free_begin=self.used, blocks_taken=used)
        S.kv_copy_blocks(self.cache, src, dst, tokens)
        self.table, self.lens, self.held, self.refs, self.used = table, lens, held, refs, used

    def compact(self):
        """All blocks in use to the front of the pool; how many there are."""
        n, most = self.n_blocks, self.n_blocks // 2
        refs, where, src, dst, counts = self.zeros(n), self.zeros(n), self.zeros(most), self.zeros(most), self.zeros(3)
        S.kv_compact(self.refs, -1, self.lens, self.table, self.bs, self.table, refs, where, src, dst, counts, held_blocks=self.held,
                     workspace=self.space)
        S.kv_copy_blocks(self.cache, src, dst)
        self.refs = refs
        self.count()
        return int(counts[0])


class Search:
    """The sessions' beams on the host: what each has emitted, and the continuations that have ended."""

    def __init__(self, prompts, beams, end):
        self.beams, self.end = beams, end
        self.histories = [[[]] for _ in prompts]        # per session and beam: tokens behind the prompt
        self.ended = [[] for _ in prompts]              # (score per token, tokens)

    def step(self, parents, tokens, scores, ends):
        """Takes over what a selection chose; ``parents`` counts the rows of all sessions."""
        rows = [(s, h) for s, hs in enumerate(self.histories) for h in hs]
        for (s, h), score in zip(rows, ends):
            if score > -float("inf"):
                self.ended[s].append((score / (len(h) + 1), h + [self.end]))
        chosen = [[] for _ in self.histories]
        for i, (p, t) in enumerate(zip(parents, tokens)):
            chosen[i // self.beams].append(rows[p][1] + [t])
        self.histories, self.scores = chosen, [scores[s * self.beams:(s + 1) * self.beams] for s in range(len(chosen))]

    def best(self):
        """Per session the best sequence by score per token, those that have not ended among them."""
        every = [e + [(x / len(h), h) for x, h in zip(xs, hs)] for e, xs, hs in zip(self.ended, self.scores, self.histories)]
        return [max(c)[1] for c in every]


def search(model, prompts, beams, n_tokens, end, block_size=16, compact_every=5):
    """Beam search with the paged cache; returns the best sequence of every session, all final beams, and the blocks in use after
    each compaction."""
    n, far = len(prompts), max(map(len, prompts))
    pages, state, packed = Pages(model, n * beams, far + n_tokens + 2, block_size), Search(prompts, beams, end), []
    pages.rows(n)
    tokens, new = i32([t for p in prompts for t in p]), [len(p) for p in prompts]
    scores = torch.zeros(n, device=DEV)
    cu_rows, cu_next = i32(list(range(n + 1))), i32([beams * s for s in range(n + 1)])
    host_lens = [0] * n
    for step in range(n_tokens):
        cu, slots = pages.places(new)
        longest, rows = max(host_lens), len(new)
        size = S.prefix_prefill_attn_workspace_bytes(pages.cache, rows, model.hq, sum(new), max(new), longest)
        workspace = torch.empty(size, dtype=torch.uint8, device=DEV) if size else None

        def attend(layer, q, k, v):
            out = torch.empty_like(q)
            S.prefix_prefill_attn(pages.cache, layer, q, k, v, out, cu, pages.lens, pages.table, max(new), longest, model.d ** -0.5,
                                  workspace)
            return out
        positions = i32([l + i for l, m in zip(host_lens, new) for i in range(m)])
        logits, k_new, v_new = model.logits(tokens, positions, attend, cu[1:].long() - 1)
        S.kv_commit(pages.cache, k_new, v_new, torch.arange(sum(new), dtype=torch.int32, device=DEV), slots)
        pages.lens = pages.lens + i32(new)
        host_lens = [l + m for l, m in zip(host_lens, new)]

        total = n * beams
        parents, tokens, best = pages.zeros(total), pages.zeros(total), torch.zeros(total, device=DEV)
        ends = torch.empty(rows, device=DEV)
        space = torch.empty(S.beam_select_workspace_bytes(*logits.shape, beams), dtype=torch.uint8, device=DEV)
        S.beam_select(logits, scores, cu_rows, cu_next, beams, parents, tokens, best, end_token=end, end_scores=ends, workspace=space)
        pages.count(taken=True)
        pages.fork(parents)
        state.step(parents.tolist(), tokens.tolist(), best.tolist(), ends.tolist())
        host_lens = [host_lens[p] for p in parents.tolist()]
        scores, cu_rows, new = best, cu_next, [1] * total
        if compact_every and step % compact_every == compact_every - 1:
            packed.append(pages.compact())
    return state.best(), state.histories, packed


def search_without_cache(model, prompts, beams, n_tokens, end):
    """The same search with every beam's whole sequence through the model in each step, and elementary operations."""
    state = Search(prompts, beams, end)
    scores = [[0.0] for _ in prompts]
    for _ in range(n_tokens):
        parents, tokens, best, ends, row = [], [], [], [], 0
        for s, prompt in enumerate(prompts):
            found = []
            for b, h in enumerate(state.histories[s]):
                logits = whole_sequence(model, prompt + h)
                x = torch.log_softmax(logits.double(), dim=-1) + scores[s][b]
                found.append(x.cpu())
            flat = torch.cat(found)
            vocab = found[0].numel()
            order = torch.argsort(flat, descending=True, stable=True)
            first = set(order[:beams].tolist())
            ends += [flat[b * vocab + end].item() if b * vocab + end in first else -float("inf") for b in range(len(found))]
            going = order[order % vocab != end][:beams]
            parents += [row + int(i) // vocab for i in going]
            tokens += [int(i) % vocab for i in going]
            best += flat[going].float().tolist()
            row += len(found)
        state.step(parents, tokens, best, ends)
        scores = state.scores
    return state.best(), state.histories


def whole_sequence(model, tokens):
    """Logits behind the last token, attention in elementary operations."""
    t = len(tokens)
    mask = torch.ones((t, t), dtype=torch.bool, device=DEV).triu(1)

    def attend(layer, q, k, v):
        g = model.hq // model.hkv
        k, v = (x.float().repeat_interleave(g, dim=1).transpose(0, 1).contiguous() for x in (k, v))
        x = torch.matmul(q.float().transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) * model.d ** -0.5
        return torch.matmul(torch.softmax(x.masked_fill(mask, -float("inf")), dim=-1), v).transpose(0, 1).to(q.dtype)
    return model.logits(i32(tokens), torch.arange(t, dtype=torch.int32, device=DEV), attend, [t - 1])[0][0]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--sessions", type=int, default=3)
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=37, help="tokens of the longest prompt")
    ap.add_argument("--tokens", type=int, default=24, help="tokens to generate per session")
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    a = ap.parse_args(argv)
    model = Scorer(dtype=torch.float32 if a.dtype == "fp32" else torch.bfloat16)
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randint(0, 512, (max(1, a.prompt - 5 * s),), generator=g).tolist() for s in range(a.sessions)]
    best, _, packed = search(model, prompts, a.beams, a.tokens, end=7)
    plain, _ = search_without_cache(model, prompts, a.beams, a.tokens, end=7)
    same = sum(x == y for x, y in zip(best, plain))
    apart = -(-(a.prompt + a.tokens) // 16) * a.beams * a.sessions
    print(f"blocks in use when packed: {packed}; without sharing up to {apart}")
    print(f"{same} of {a.sessions} sessions have the same best sequence with the cache and without", flush=True)
    return 0 if same == a.sessions or a.dtype == "bf16" else 1


if __name__ == "__main__":
    raise SystemExit(main())
