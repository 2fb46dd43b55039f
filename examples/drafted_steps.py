"""Speculative decoding over the paged cache: the operators of a drafted step, run together by a small model with random weights.

    python examples/drafted_steps.py [--sessions 4] [--tokens 96] [--dtype bf16]

Every session decodes greedily.  A step drafts a tree of tokens for each of them: what followed earlier occurrences of the
session's last tokens in its own history, continuations with a common beginning sharing nodes.  One pass of the model scores
all nodes of all trees at once, the path that agrees with the model is kept and goes into the cache:

    build_tables   cache blocks and slots for the drafted tokens, from the free list
    tree_mask      who sees whom, and positions
    tree_attn      per layer: [paged cache ; the tree under its mask]
    tree_accept    the path that agrees, the token behind it, the new lengths
    kv_commit      the path's K,V rows of all layers into their slots

Blocks that a step took for nodes that were not accepted stay with their session and hold its next tokens.  The script decodes
the same prompts with trees of one node as well and compares: the tokens have to be the same (in bf16 a near tie may
fall the other way, since sums run in another order).
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2412_16434_amd as S  # noqa: E402

DEV = "cuda:0"


class Model:
    """Embedding, layers of grouped-query attention with rotary positions and a gated product, tied output."""

    def __init__(self, layers=4, hidden=256, n_q_heads=8, n_kv_heads=2, head_dim=64, vocab=512, dtype=torch.float32, seed=0):
        g = torch.Generator().manual_seed(seed)
        w = lambda a, b: (torch.randn((a, b), generator=g) / a ** 0.5).to(dtype).to(DEV)  # noqa: E731
        self.layers, self.hq, self.hkv, self.d, self.dtype = layers, n_q_heads, n_kv_heads, head_dim, dtype
        self.embed = w(vocab, hidden) * vocab ** 0.5
        self.wq, self.wk, self.wv, self.wo, self.up, self.gate, self.down = (
            [w(*shape) for _ in range(layers)] for shape in (
                (hidden, n_q_heads * head_dim), (hidden, n_kv_heads * head_dim), (hidden, n_kv_heads * head_dim),
                (n_q_heads * head_dim, hidden), (hidden, 2 * hidden), (hidden, 2 * hidden), (2 * hidden, hidden)))
        self.inv_freq = 10000.0 ** (-torch.arange(0, head_dim, 2, device=DEV, dtype=torch.float32) / head_dim)

    @staticmethod
    def norm(x):
        return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def rotate(self, x, positions):
        angle = positions.float()[:, None, None] * self.inv_freq
        a, b = x.float().chunk(2, dim=-1)
        return torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], dim=-1).to(x.dtype)

    def forward(self, tokens, positions, attend):
        """Tokens the model puts behind each of ``tokens`` and the K,V rows of all layers; ``attend(layer, q, k, v)`` is the
        attention."""
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
        return (self.norm(x).float() @ self.embed.float().T).argmax(-1).int(), k_new, v_new


class Server:
    """The paged cache of some sessions and a step over all of them."""

    def __init__(self, model, n_sessions, max_tokens, block_size=16):
        self.model, self.bs = model, block_size
        per_session = -(-max_tokens // block_size) + 1
        self.n_blocks = n_sessions * per_session
        pool = lambda: torch.zeros((model.layers, self.n_blocks, block_size, model.hkv, model.d), dtype=model.dtype,  # noqa: E731
                                   device=DEV)
        self.cache = S.KVCache(pool(), pool())
        self.table = self.i32(n_sessions, per_session).fill_(-1)
        self.free = torch.randperm(self.n_blocks, generator=torch.Generator().manual_seed(1)).int().to(DEV)
        # (two of each: a call reads one and writes the other)
        self.used, self.held = [self.i32(1), self.i32(1)], [self.i32(n_sessions), self.i32(n_sessions)]
        self.lens, self.host_lens = self.i32(n_sessions), [0] * n_sessions  # cached tokens, and the host's copy
        self.workspace = None

    @staticmethod
    def i32(*shape):
        return torch.zeros(shape, dtype=torch.int32, device=DEV)

    def _tables(self, new_lens):
        """Blocks for the new tokens of every session: (cu_new_lens, slot map)."""
        total, n = sum(new_lens), len(new_lens)
        cu, slots = self.i32(n + 1), torch.empty(total, dtype=torch.int64, device=DEV)
        S.build_tables(self.lens, torch.tensor(new_lens, dtype=torch.int32).to(DEV), self.table, self.free, self.bs, self.n_blocks,
                       total, cu_new_lens=cu, slot_map=slots, blocks_taken=self.used[1], held_blocks=self.held[0],
                       held_after=self.held[1], free_begin=self.used[0])
        self.used.reverse()
        self.held.reverse()
        return cu, slots

    def prompts(self, prompts):
        """All prompts into the cache; the token behind each."""
        m, lens = self.model, [len(p) for p in prompts]
        total, far = sum(lens), max(lens)
        cu, slots = self._tables(lens)
        tokens = torch.tensor([t for p in prompts for t in p], dtype=torch.int32).to(DEV)
        positions = torch.cat([torch.arange(n) for n in lens]).int().to(DEV)
        scale = m.d ** -0.5
        size = S.prefix_prefill_attn_workspace_bytes(self.cache, len(prompts), m.hq, total, far, 0)
        workspace = torch.empty(size, dtype=torch.uint8, device=DEV) if size else None

        def attend(layer, q, k, v):
            out = torch.empty_like(q)
            S.prefix_prefill_attn(self.cache, layer, q, k, v, out, cu, self.lens, self.table, far, 0, scale, workspace)
            return out
        target, k_new, v_new = m.forward(tokens, positions, attend)
        S.kv_commit(self.cache, k_new, v_new, torch.arange(total, dtype=torch.int32, device=DEV), slots)
        self.lens = torch.tensor(lens, dtype=torch.int32).to(DEV)
        self.host_lens = lens
        return target[cu[1:].long() - 1].tolist()

    def step(self, trees):
        """One step; ``trees``: per session (tokens, parents), the first node being the session's last token, which is not
        cached yet.  Returns per session the indices of its accepted nodes and the token behind them."""
        m, n, longest = self.model, len(trees), max(self.host_lens)
        sizes = [len(t) for t, _ in trees]
        total, most = sum(sizes), max(sizes)
        draft = torch.tensor([t for tokens, _ in trees for t in tokens], dtype=torch.int32).to(DEV)
        parents = torch.tensor([p for _, links in trees for p in links], dtype=torch.int32).to(DEV)
        cu, slots = self._tables(sizes)
        mask = torch.empty((total, -(-most // 64)), dtype=torch.int64, device=DEV)
        positions = self.i32(total)
        S.tree_mask(parents, cu, most, mask, prefix_lens=self.lens, positions=positions)

        size = S.tree_attn_workspace_bytes(self.cache, n, m.hq, total, most, longest)
        if size and (self.workspace is None or self.workspace.numel() < size):
            self.workspace = torch.empty(size, dtype=torch.uint8, device=DEV)

        def attend(layer, q, k, v):
            out = torch.empty_like(q)
            S.tree_attn(self.cache, layer, q, k, v, out, mask, cu, self.lens, self.table, most, longest, m.d ** -0.5,
                        self.workspace)
            return out
        target, k_new, v_new = m.forward(draft, positions, attend)
        rows, count, following, lens = self.i32(total), self.i32(n), self.i32(n), self.i32(n)
        S.tree_accept(draft, parents, target, cu, self.lens, rows, count, following, lens)
        # The t-th token of a session's path goes where the t-th of its drafted tokens would have gone
        S.kv_commit(self.cache, k_new, v_new, rows, slots)
        self.lens = lens
        cu_h, rows_h, count_h, following_h = (x.tolist() for x in (cu, rows, count, following))
        self.host_lens = [a + b for a, b in zip(self.host_lens, count_h)]
        return [[r - cu_h[s] for r in rows_h[cu_h[s]:cu_h[s] + count_h[s]]] for s in range(n)], following_h


def draft_from_history(history, branches, depth):
    """A tree over ``history``'s last token: what followed up to ``branches`` earlier occurrences of its last two tokens (else of
    the last one), ``depth`` tokens each."""
    tokens, parents, children = [history[-1]], [-1], {}
    for context in (2, 1):
        if branches == 0 or len(tokens) > 1:
            break
        tail, found = history[-context:], 0
        for at in range(len(history) - context - 1, -1, -1):
            if found == branches:
                break
            if history[at:at + context] != tail:
                continue
            found += 1
            node = 0
            for t in history[at + context:at + context + depth]:
                if (node, t) not in children:
                    children[node, t] = len(tokens)
                    tokens.append(t)
                    parents.append(node)
                node = children[node, t]
    return tokens, parents


def generate(model, prompts, n_tokens, branches=4, depth=7, block_size=16):
    """``n_tokens`` tokens behind every prompt; returns them and the number of steps.  ``branches`` 0: one token a step."""
    reserve = 1 + branches * depth
    server = Server(model, len(prompts), max(map(len, prompts)) + n_tokens + 2 * reserve, block_size)
    history = [list(p) + [t] for p, t in zip(prompts, server.prompts(prompts))]
    steps = 0
    while min(len(h) - len(p) for h, p in zip(history, prompts)) < n_tokens:
        # (a session that is done goes on with no tree until all are)
        trees = []
        for h, p in zip(history, prompts):
            left = n_tokens - (len(h) - len(p))
            trees.append(draft_from_history(h, branches, min(depth, left)) if left > 0 else ([], []))
        paths, following = server.step(trees)
        for h, (tokens, _), path, token in zip(history, trees, paths, following):
            if tokens:
                h += [tokens[i] for i in path[1:]] + [token]
        steps += 1
    return [h[len(p):len(p) + n_tokens] for h, p in zip(history, prompts)], steps


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--sessions", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=40, help="tokens of the longest prompt")
    ap.add_argument("--tokens", type=int, default=96, help="tokens to generate per session")
    ap.add_argument("--branches", type=int, default=4)
    ap.add_argument("--depth", type=int, default=7)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    a = ap.parse_args(argv)
    model = Model(dtype=torch.float32 if a.dtype == "fp32" else torch.bfloat16)
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randint(0, 512, (max(1, a.prompt - 3 * s),), generator=g).tolist() for s in range(a.sessions)]
    results = []
    for branches in (0, a.branches):
        generate(model, prompts, min(a.tokens, 8), branches, a.depth)  # (libraries and kernels are loaded)
        torch.cuda.synchronize()
        start = time.perf_counter()
        tokens, steps = generate(model, prompts, a.tokens, branches, a.depth)
        results.append(tokens)
        print(f"{'trees' if branches else 'one token a step'}: {steps} steps, {1e3 * (time.perf_counter() - start):.1f} ms, "
              f"{a.sessions * a.tokens / steps:.2f} tokens per step", flush=True)
    same = sum(x == y for x, y in zip(*results))
    print(f"{same} of {a.sessions} sessions have the same tokens both ways", flush=True)
    return 0 if same == a.sessions or a.dtype == "bf16" else 1


if __name__ == "__main__":
    raise SystemExit(main())
