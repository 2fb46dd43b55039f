"""symph_kv_copy_blocks with long lists (more than 2^17 pieces: pairs, layers, K and V), valid pairs all over or everywhere: both widths
of access, filled slots, few and many layers."""
import numpy as np
import pytest
import torch

import paper_2412_16434_amd as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def _pools(layers, n_blocks, bs, hkv, d, dtype, pad, seed):
    """Random bits, `pad` elements behind every block."""
    width, block = {torch.bfloat16: torch.int16, torch.float32: torch.int32}[dtype], bs * hkv * d
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    raw = [torch.randint(-30000, 30000, (layers, n_blocks, block + pad), generator=g, dtype=width, device=DEV) for _ in range(2)]
    shape, strides = (layers, n_blocks, bs, hkv, d), (n_blocks * (block + pad), block + pad, hkv * d, d, 1)
    return S.KVCache(*(r.view(dtype).as_strided(shape, strides) for r in raw)), raw


# layers, entries of the list, valid pairs of them, tokens of a block, heads, head size, elements behind a block.  A group is 64 entries:
# many workgroups to a group of one layer (32), three, and one; rows of 16-byte vectors and of 4-byte words
CASES = [(2, 70_000, 70, 16, 1, 64, 0), (2, 70_000, 2000, 5, 1, 6, 2), (1, 65_600, 3000, 16, 2, 8, 8), (33, 2000, 1900, 3, 1, 10, 0),
         (33, 2047, 2047, 4, 3, 8, 0), (700, 3830, 3000, 1, 1, 2, 0), (700, 3830, 3830, 2, 1, 8, 8), (2100, 2048, 2048, 1, 1, 2, 0),
         (4200, 2048, 1500, 1, 1, 8, 0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layers,entries,valid,bs,hkv,d,pad", CASES)
def test_long_lists(layers, entries, valid, bs, hkv, d, pad, dtype):
    assert 2 * entries * layers > 1 << 17
    n, rs = 2 * valid + 3, np.random.RandomState(entries + valid)
    cache, raw = _pools(layers, n, bs, hkv, d, dtype, pad, valid)
    ids = rs.permutation(n)
    src = rs.choice([-1, -2 ** 31, n, 2 ** 31 - 1], size=entries)      # (nothing of a pair that is not there is copied)
    dst = np.where(rs.random_sample(entries) < 0.5, -1, n)
    at = np.sort(rs.permutation(entries)[:valid])
    src[at], dst[at] = ids[:valid], ids[valid:2 * valid]
    half = at[rs.random_sample(valid) < 0.1]
    src[half[::3]], dst[half[1::3]] = -1, n                            # one side only
    dst[half[2::3]] = src[half[2::3]]                                  # a block to itself
    tokens = rs.randint(-2, bs + 3, size=entries)
    there = (src >= 0) & (src < n) & (dst >= 0) & (dst < n)
    row = hkv * d
    for filled in (tokens, None):
        want = [r.clone() for r in raw]
        count = np.full(entries, bs) if filled is None else np.clip(filled, 0, bs)
        for t in range(bs):
            copied = there & (count > t)
            a, b = (torch.from_numpy(x[copied]).to(DEV) for x in (src, dst))
            for w in want:
                w[:, b, t * row:(t + 1) * row] = w[:, a, t * row:(t + 1) * row]
        S.kv_copy_blocks(cache, _i32(src), _i32(dst), None if filled is None else _i32(filled))
        torch.cuda.synchronize()
        assert torch.equal(raw[0], want[0]) and torch.equal(raw[1], want[1])
