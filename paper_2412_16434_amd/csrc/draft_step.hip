// What surrounds the attention of a speculative decoding step: block tables and slot maps from lengths, ancestor masks of
// the drafted trees, the accepted path, and its K,V rows into the paged cache.  The first three are a handful of dependent
// trips to memory per session (their bytes take less than a launch does up to some thousand sessions); the last one, and
// tables for whole arriving sessions, write HBM.
#include "common.h"

namespace symph {

static int log2_or_neg(int64_t x) { return (x > 0 && (x & (x - 1)) == 0) ? __builtin_ctzll((unsigned long long)x) : -1; }

// ---- block tables and slot maps ----------------------------------------------------------------------------------
struct TablesParams {
  const int32_t* prefix_lens;
  const int32_t* new_lens;
  const int32_t* held;
  int32_t* table;
  const int32_t* free_blocks;
  const int32_t* free_begin;
  int32_t* cu_new_lens;
  int64_t* token_offsets;
  int64_t* slot_map;
  int32_t* positions;
  int32_t* blocks_taken;
  int32_t* held_after;
  int64_t total;
  int32_t n_sessions, table_stride, n_free, block_size, bs_shift, n_blocks;
};

constexpr int kTabThreads = 256, kTabSess = 4;             // sessions a thread adds up at a time
constexpr int kTabChunk = kTabThreads * kTabSess;
constexpr int kTabTokens = 4;                              // consecutive tokens of a thread: 16- and 32-byte stores

__device__ __forceinline__ int64_t wave_scan64(int64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t up = __shfl_up((long long)v, o);
    if (lane >= o) v += up;
  }
  return v;
}

// Every workgroup owns kTabThreads * kTabTokens consecutive new tokens and adds up the lengths of the sessions itself, up to
// the one its tokens end in (64-bit sums: nothing has to be handed over, one launch).  A table entry is written by the
// thread that has the first token of its block.  One more workgroup writes what there is per session.
__global__ __launch_bounds__(kTabThreads) void build_tables_kernel(const TablesParams p) {
  __shared__ int64_t first_tok[kTabChunk + 1], first_blk[kTabChunk];  // relative to the chunk's first session
  __shared__ int32_t prefix[kTabChunk], held[kTabChunk];
  __shared__ int64_t wave_sums[kTabThreads / 64][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool per_session = blockIdx.x == gridDim.x - 1;
  const int64_t t_begin = (int64_t)blockIdx.x * (kTabThreads * kTabTokens);
  const int64_t t_end = min(p.total, t_begin + kTabThreads * kTabTokens);
  const int64_t t0 = t_begin + tid * kTabTokens;
  const unsigned bs = (unsigned)p.block_size;
  auto block_of = [&](unsigned pos) { return p.bs_shift >= 0 ? pos >> p.bs_shift : pos / bs; };
  auto blocks_for = [&](unsigned n) { return n == 0 ? 0u : block_of(n - 1) + 1; };
  const int64_t free_begin = p.free_begin ? (int64_t)p.free_begin[0] : 0;

  int64_t slots[kTabTokens];
  int32_t pos_of[kTabTokens];
#pragma unroll
  for (int k = 0; k < kTabTokens; ++k) slots[k] = -1, pos_of[k] = -1;
  int64_t run_tok = 0, run_blk = free_begin;
  for (int c0 = 0; c0 < p.n_sessions; c0 += kTabChunk) {
    unsigned P[kTabSess], N[kTabSess], H[kTabSess], need[kTabSess];
    int64_t tok = 0, blk = 0;
#pragma unroll
    for (int k = 0; k < kTabSess; ++k) {
      const int i = c0 + tid * kTabSess + k;
      const bool in = i < p.n_sessions;
      P[k] = in ? (unsigned)max(p.prefix_lens[i], 0) : 0u;
      N[k] = in ? (unsigned)max(p.new_lens[i], 0) : 0u;
      H[k] = in && p.held ? (unsigned)max(p.held[i], 0) : 0u;
    }
#pragma unroll
    for (int k = 0; k < kTabSess; ++k) {
      H[k] = max(H[k], blocks_for(P[k]));
      const unsigned all = blocks_for(P[k] + N[k]);  // (two values below 2^31: fits 32 bits)
      need[k] = all > H[k] ? all - H[k] : 0u;
      tok += N[k];
      blk += need[k];
    }
    const int64_t tok_incl = wave_scan64(tok), blk_incl = wave_scan64(blk);
    if (lane == 63) {
      wave_sums[wave][0] = tok_incl;
      wave_sums[wave][1] = blk_incl;
    }
    __syncthreads();
    int64_t tok_at = tok_incl - tok, blk_at = blk_incl - blk, chunk_tok = 0, chunk_blk = 0;
#pragma unroll
    for (int w = 0; w < kTabThreads / 64; ++w) {
      if (w < wave) {
        tok_at += wave_sums[w][0];
        blk_at += wave_sums[w][1];
      }
      chunk_tok += wave_sums[w][0];
      chunk_blk += wave_sums[w][1];
    }
#pragma unroll
    for (int k = 0; k < kTabSess; ++k) {
      const int at = tid * kTabSess + k, i = c0 + at;
      first_tok[at] = tok_at;
      first_blk[at] = blk_at;
      prefix[at] = (int32_t)P[k];
      held[at] = (int32_t)H[k];
      if (per_session && i < p.n_sessions) {
        if (p.cu_new_lens) p.cu_new_lens[i] = (int32_t)(run_tok + tok_at);
        if (p.token_offsets) p.token_offsets[i] = run_tok + tok_at;
        if (p.held_after) p.held_after[i] = (int32_t)(H[k] + need[k]);
      }
      tok_at += N[k];
      blk_at += need[k];
    }
    if (tid == kTabThreads - 1) first_tok[kTabChunk] = chunk_tok;
    __syncthreads();
    if (!per_session && run_tok + chunk_tok > t_begin) {
      int s = -1;  // session of the present token, relative to the chunk
#pragma unroll
      for (int k = 0; k < kTabTokens; ++k) {
        const int64_t t = t0 + k - run_tok;
        if (t < 0 || t >= chunk_tok || t0 + k >= t_end) continue;
        if (s < 0) {  // the last session that begins at or before t (those without tokens begin where the next one does)
          int lo = 0, hi = kTabChunk;
          while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first_tok[mid] <= t)
              lo = mid;
            else
              hi = mid;
          }
          s = lo;
        }
        while (first_tok[s + 1] <= t) ++s;
        const unsigned pos = (unsigned)prefix[s] + (unsigned)(t - first_tok[s]);
        const unsigned b = block_of(pos), place = pos - b * bs;
        int32_t id = -1;
        if (b < (unsigned)p.table_stride) {
          int32_t* const entry = p.table + (int64_t)(c0 + s) * p.table_stride + b;
          if (b >= (unsigned)held[s]) {
            const int64_t j = run_blk + first_blk[s] + (b - (unsigned)held[s]);
            if (j >= 0 && j < p.n_free) id = p.free_blocks[j];
            if (place == 0) *entry = id;
          } else
            id = *entry;
        }
        slots[k] = id >= 0 && id < p.n_blocks ? (int64_t)id * bs + place : -1;
        pos_of[k] = (int32_t)pos;
      }
    }
    run_tok += chunk_tok;
    run_blk += chunk_blk;
    if (!per_session && run_tok >= t_end) break;
    __syncthreads();  // (the next chunk's sums go where this one's are read)
  }
  if (per_session) {
    if (tid == 0) {
      if (p.cu_new_lens) p.cu_new_lens[p.n_sessions] = (int32_t)run_tok;
      if (p.token_offsets) p.token_offsets[p.n_sessions] = run_tok;
      if (p.blocks_taken) p.blocks_taken[0] = (int32_t)min(run_blk, (int64_t)0x7FFFFFFF);
    }
    return;
  }
  typedef long long i64x2 __attribute__((ext_vector_type(2)));
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  if (p.slot_map) {
    if (t0 + kTabTokens <= t_end && ((uintptr_t)p.slot_map & 15) == 0) {
      *reinterpret_cast<i64x2*>(p.slot_map + t0) = i64x2{slots[0], slots[1]};
      *reinterpret_cast<i64x2*>(p.slot_map + t0 + 2) = i64x2{slots[2], slots[3]};
    } else {
#pragma unroll
      for (int k = 0; k < kTabTokens; ++k)
        if (t0 + k < t_end) p.slot_map[t0 + k] = slots[k];
    }
  }
  if (p.positions) {
    if (t0 + kTabTokens <= t_end && ((uintptr_t)p.positions & 15) == 0) {
      *reinterpret_cast<i32x4*>(p.positions + t0) = i32x4{pos_of[0], pos_of[1], pos_of[2], pos_of[3]};
    } else {
#pragma unroll
      for (int k = 0; k < kTabTokens; ++k)
        if (t0 + k < t_end) p.positions[t0 + k] = pos_of[k];
    }
  }
}

// ---- masks of trees ----------------------------------------------------------------------------------------------
struct TreeMaskParams {
  const int32_t* parents;
  const int32_t* cu_new_lens;
  const int32_t* prefix_lens;
  uint64_t* mask;
  int32_t* positions;
  int32_t total, max_new, words;
};

// A session's nodes in chunks of 64, a node per lane.  Inside a chunk the ancestors follow from six rounds of pointer
// doubling between lanes; the ancestor with the lowest index leads out of the chunk through its parent (a parent comes
// before its children).  What a row has in earlier chunks is then found by one walk over chunks, not over ancestors.
__global__ __launch_bounds__(256) void tree_mask_kernel(const TreeMaskParams p) {
  extern __shared__ __attribute__((aligned(16))) char tree_lds[];
  const int cap = (p.max_new + 63) & ~63;
  uint64_t* const in_chunk = reinterpret_cast<uint64_t*>(tree_lds);      // ancestors (and self) inside the node's chunk
  int32_t* const way_out = reinterpret_cast<int32_t*>(in_chunk + cap);  // first ancestor before the chunk, -1: none
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
  const int cu = max(p.cu_new_lens[s], 0);
  const int n = min(min(p.cu_new_lens[s + 1], p.total) - cu, p.max_new);
  const int row0 = blockIdx.y * blockDim.x;
  if (row0 >= n) return;
  const int row_end = min(n, row0 + (int)blockDim.x);
  for (int c = wave; c * 64 < row_end; c += waves) {
    const int i = c * 64 + lane;
    int par = i < n ? p.parents[cu + i] : -1;
    if (par < 0 || par >= i) par = -1;
    int jump = par >= c * 64 ? par - c * 64 : -1;
    unsigned long long bits = 1ull << lane;
#pragma unroll
    for (int r = 0; r < 6; ++r) {
      const int from = jump < 0 ? lane : jump;
      bits |= __shfl(bits, from);
      const int next = __shfl(jump, from);
      if (jump >= 0) jump = next;
    }
    in_chunk[i] = bits;
    way_out[i] = __shfl(par, __builtin_ctzll(bits));
  }
  __syncthreads();
  const int i = row0 + tid;
  if (i >= row_end) return;
  uint64_t* const row = p.mask + (int64_t)(cu + i) * p.words;
  int x = i, seen = 0;
  for (int w = p.words - 1; w >= 0; --w) {
    uint64_t bits = 0;
    if (x >= 0 && (x >> 6) == w) {
      bits = in_chunk[x];
      x = way_out[x];
      seen += __popcll(bits);
    }
    row[w] = bits;
  }
  if (p.positions) p.positions[cu + i] = (p.prefix_lens ? p.prefix_lens[s] : 0) + seen - 1;
}

// ---- the accepted path -------------------------------------------------------------------------------------------
struct AcceptParams {
  const int32_t* draft;
  const int32_t* parents;
  const int32_t* target;
  const int32_t* cu_new_lens;
  const int32_t* prefix_lens;
  int32_t* rows;
  int32_t* n_accepted;
  int32_t* next_tokens;
  int32_t* new_prefix_lens;
  int32_t n_sessions, total;
};

// A wave per session, 64 nodes at a time.  Which nodes agree with their parent's target token is known at once; the walk then
// only asks the lanes: the lowest one whose parent is the present node.  Children come after their parents, so one pass is
// enough.
__global__ __launch_bounds__(256) void tree_accept_kernel(const AcceptParams p) {
  const int lane = threadIdx.x & 63;
  const int s = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (s >= p.n_sessions) return;
  const int cu = max(p.cu_new_lens[s], 0);
  const int n = max(min(p.cu_new_lens[s + 1], p.total) - cu, 0);
  const int P = p.prefix_lens ? p.prefix_lens[s] : 0;
  int node = 0, count = n > 0 ? 1 : 0;
  for (int c = 0; c < n; c += 64) {
    const int i = c + lane;
    int par = i < n ? p.parents[cu + i] : -1;
    if (par < 0 || par >= i) par = -1;
    const bool agrees = par >= 0 && p.draft[cu + i] == p.target[cu + par];
    int mine = i == 0 && n > 0 ? 0 : -1;  // this node's place on the path
    for (;;) {
      const uint64_t next = __ballot(agrees && par == node && i > node);
      if (next == 0) break;
      const int at = __builtin_ctzll(next);
      node = c + at;
      if (lane == at) mine = count;
      ++count;
    }
    if (mine >= 0) p.rows[cu + mine] = cu + i;
  }
  for (int k = count + lane; k < n; k += 64) p.rows[cu + k] = -1;
  if (lane == 0) {
    p.n_accepted[s] = count;
    p.next_tokens[s] = n > 0 ? p.target[cu + node] : -1;
    if (p.new_prefix_lens) p.new_prefix_lens[s] = P + count;
  }
}

// ---- rows of all layers through a slot map -----------------------------------------------------------------------
struct CommitParams {
  char* k_base;
  char* v_base;
  const char* k_new;
  const char* v_new;
  const int32_t* rows;
  const int64_t* slot_map;
  int64_t layer_stride_b, block_stride_b, new_layer_b;
  int32_t row_bytes, vecs_per_row, block_size, bs_shift, n_blocks, n_rows, n_entries;
};

// A workgroup has 64 entries of one layer.  Most of them are skipped (a tree has many nodes and one path), so the entries that
// are written are counted off first, one per lane, and the waves take them in turn, K and V of a row together.
template <typename VecT>
__global__ __launch_bounds__(256) void kv_commit_kernel(const CommitParams p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int t = blockIdx.x * 64 + lane;
  int32_t row = -1;
  int64_t dst = 0;
  if (t < p.n_entries) {
    row = p.rows[t];
    const int64_t slot = p.slot_map[t];
    if (row >= p.n_rows || slot < 0) row = -1;
    if (row >= 0) {
      const int64_t b = p.bs_shift >= 0 ? slot >> p.bs_shift : slot / p.block_size;
      if (b < p.n_blocks)
        dst = b * p.block_stride_b + (slot - b * p.block_size) * p.row_bytes;
      else
        row = -1;
    }
  }
  const uint64_t valid = __ballot(row >= 0);
  const int64_t layer_b = (int64_t)blockIdx.y * p.layer_stride_b, new_b = (int64_t)blockIdx.y * p.new_layer_b;
  int turn = 0;
  for (uint64_t left = valid; left; left &= left - 1) {
    if ((turn++ & 3) != wave) continue;
    const int at = __builtin_ctzll(left);
    const int64_t src = (int64_t)__builtin_amdgcn_readlane(row, at) * p.row_bytes + new_b;
    const int64_t to = ((int64_t)__builtin_amdgcn_readlane((int)(dst >> 32), at) << 32 |
                        (uint32_t)__builtin_amdgcn_readlane((int)dst, at)) + layer_b;
    for (int v = lane; v < p.vecs_per_row; v += 64) {
      const VecT k = reinterpret_cast<const VecT*>(p.k_new + src)[v], x = reinterpret_cast<const VecT*>(p.v_new + src)[v];
      reinterpret_cast<VecT*>(p.k_base + to)[v] = k;
      reinterpret_cast<VecT*>(p.v_base + to)[v] = x;
    }
  }
}

}  // namespace symph

using namespace symph;

extern "C" {

int32_t symph_build_tables(const int32_t* d_prefix_lens, const int32_t* d_new_lens, const int32_t* d_held_blocks,
                           int32_t n_sessions, int32_t* d_block_table, int32_t table_stride, const int32_t* d_free_blocks,
                           int32_t n_free, const int32_t* d_free_begin, int32_t block_size, int32_t n_blocks,
                           int64_t total_new_tokens, int32_t* d_cu_new_lens, int64_t* d_token_offsets, int64_t* d_slot_map,
                           int32_t* d_positions, int32_t* d_blocks_taken, int32_t* d_held_after, void* stream) {
  if (n_sessions < 0 || table_stride < 0 || n_free < 0 || block_size <= 0 || n_blocks <= 0 || total_new_tokens < 0)
    return SYMPH_EINVAL;
  if (n_sessions > 0 && (!d_prefix_lens || !d_new_lens)) return SYMPH_EINVAL;
  if (n_sessions > 0 && total_new_tokens > 0 && (!d_block_table || table_stride == 0)) return SYMPH_EINVAL;
  if (n_free > 0 && !d_free_blocks) return SYMPH_EINVAL;
  if (d_cu_new_lens && total_new_tokens > 0x7FFFFFFFLL) return SYMPH_EINVAL;
  if ((d_held_after && d_held_after == d_held_blocks) || (d_blocks_taken && d_blocks_taken == d_free_begin)) return SYMPH_EINVAL;
  TablesParams p;
  p.prefix_lens = d_prefix_lens;
  p.new_lens = d_new_lens;
  p.held = d_held_blocks;
  p.table = d_block_table;
  p.free_blocks = d_free_blocks;
  p.free_begin = d_free_begin;
  p.cu_new_lens = d_cu_new_lens;
  p.token_offsets = d_token_offsets;
  p.slot_map = d_slot_map;
  p.positions = d_positions;
  p.blocks_taken = d_blocks_taken;
  p.held_after = d_held_after;
  p.total = total_new_tokens;
  p.n_sessions = n_sessions;
  p.table_stride = table_stride;
  p.n_free = n_free;
  p.block_size = block_size;
  p.bs_shift = log2_or_neg(block_size);
  p.n_blocks = n_blocks;
  const int64_t groups = ceil_div64(total_new_tokens, kTabThreads * kTabTokens) + 1;
  if (groups > 0x7FFFFFFFLL) return SYMPH_EUNSUPPORTED;
  hipLaunchKernelGGL(build_tables_kernel, dim3((unsigned)groups), dim3(kTabThreads), 0, (hipStream_t)stream, p);
  return hipGetLastError() == hipSuccess ? SYMPH_OK : SYMPH_ELAUNCH;
}

int32_t symph_tree_mask(const int32_t* d_parents, const int32_t* d_cu_new_lens, const int32_t* d_prefix_lens,
                        int32_t n_sessions, int32_t total_new_tokens, int32_t max_new_len, uint64_t* d_mask,
                        int32_t mask_words, int32_t* d_positions, void* stream) {
  if (n_sessions < 0 || total_new_tokens < 0 || max_new_len < 0 || mask_words < 0) return SYMPH_EINVAL;
  if (max_new_len > total_new_tokens) return SYMPH_EINVAL;
  if ((int64_t)mask_words * 64 < max_new_len) return SYMPH_EINVAL;
  if (max_new_len > SYMPH_TREE_MAX_NODES) return SYMPH_EUNSUPPORTED;
  if (n_sessions == 0 || max_new_len == 0) return SYMPH_OK;
  if (!d_parents || !d_cu_new_lens || !d_mask) return SYMPH_EINVAL;
  TreeMaskParams p;
  p.parents = d_parents;
  p.cu_new_lens = d_cu_new_lens;
  p.prefix_lens = d_prefix_lens;
  p.mask = d_mask;
  p.positions = d_positions;
  p.total = total_new_tokens;
  p.max_new = max_new_len;
  p.words = mask_words;
  const unsigned threads = max_new_len <= 64 ? 64 : 256;
  const unsigned lds = (unsigned)((max_new_len + 63) & ~63) * 12;
  hipLaunchKernelGGL(tree_mask_kernel, dim3((unsigned)n_sessions, (max_new_len + threads - 1) / threads), dim3(threads), lds,
                     (hipStream_t)stream, p);
  return hipGetLastError() == hipSuccess ? SYMPH_OK : SYMPH_ELAUNCH;
}

int32_t symph_tree_accept(const int32_t* d_draft_tokens, const int32_t* d_parents, const int32_t* d_target_tokens,
                          const int32_t* d_cu_new_lens, const int32_t* d_prefix_lens, int32_t n_sessions,
                          int32_t total_new_tokens, int32_t* d_rows, int32_t* d_n_accepted, int32_t* d_next_tokens,
                          int32_t* d_new_prefix_lens, void* stream) {
  if (n_sessions < 0 || total_new_tokens < 0) return SYMPH_EINVAL;
  if (n_sessions == 0) return SYMPH_OK;
  if (!d_cu_new_lens || !d_n_accepted || !d_next_tokens || (d_new_prefix_lens && !d_prefix_lens)) return SYMPH_EINVAL;
  if (total_new_tokens > 0 && (!d_draft_tokens || !d_parents || !d_target_tokens || !d_rows)) return SYMPH_EINVAL;
  AcceptParams p;
  p.draft = d_draft_tokens;
  p.parents = d_parents;
  p.target = d_target_tokens;
  p.cu_new_lens = d_cu_new_lens;
  p.prefix_lens = d_prefix_lens;
  p.rows = d_rows;
  p.n_accepted = d_n_accepted;
  p.next_tokens = d_next_tokens;
  p.new_prefix_lens = d_new_prefix_lens;
  p.n_sessions = n_sessions;
  p.total = total_new_tokens;
  hipLaunchKernelGGL(tree_accept_kernel, dim3((unsigned)((n_sessions + 3) / 4)), dim3(256), 0, (hipStream_t)stream, p);
  return hipGetLastError() == hipSuccess ? SYMPH_OK : SYMPH_ELAUNCH;
}

int32_t symph_kv_commit(const symph_kv_cache* cache, const void* d_k_new, const void* d_v_new, int32_t n_rows,
                        const int32_t* d_rows, const int64_t* d_slot_map, int32_t n_entries, void* stream) {
  const int32_t rc = validate_cache(cache);
  if (rc != SYMPH_OK) return rc;
  if (n_rows < 0 || n_entries < 0) return SYMPH_EINVAL;
  if (n_rows == 0 || n_entries == 0) return SYMPH_OK;
  if (!d_k_new || !d_v_new || !d_rows || !d_slot_map) return SYMPH_EINVAL;
  const int eb = elem_bytes_of(cache->dtype);
  const int64_t row_bytes = (int64_t)cache->n_kv_heads * cache->head_dim * eb;
  if (row_bytes > 0x7FFFFFFF || cache->n_layers > 65535) return SYMPH_EUNSUPPORTED;
  CommitParams p;
  p.k_base = (char*)cache->k_base;
  p.v_base = (char*)cache->v_base;
  p.k_new = (const char*)d_k_new;
  p.v_new = (const char*)d_v_new;
  p.rows = d_rows;
  p.slot_map = d_slot_map;
  p.layer_stride_b = cache->layer_stride * eb;
  p.block_stride_b = cache->block_stride * eb;
  p.new_layer_b = n_rows * row_bytes;
  const uintptr_t align_or = (uintptr_t)p.k_base | (uintptr_t)p.v_base | (uintptr_t)p.k_new | (uintptr_t)p.v_new |
                             (uintptr_t)p.layer_stride_b | (uintptr_t)p.block_stride_b | (uintptr_t)row_bytes;
  if (align_or & 3) return SYMPH_EUNSUPPORTED;
  const int vec = (align_or & 15) ? 4 : 16;
  p.row_bytes = (int32_t)row_bytes;
  p.vecs_per_row = (int32_t)(row_bytes / vec);
  p.block_size = cache->block_size;
  p.bs_shift = log2_or_neg(cache->block_size);
  p.n_blocks = cache->n_blocks;
  p.n_rows = n_rows;
  p.n_entries = n_entries;
  const dim3 grid((unsigned)(((int64_t)n_entries + 63) / 64), (unsigned)cache->n_layers);
  if (vec == 16)
    hipLaunchKernelGGL(kv_commit_kernel<u32x4>, grid, dim3(256), 0, (hipStream_t)stream, p);
  else
    hipLaunchKernelGGL(kv_commit_kernel<unsigned int>, grid, dim3(256), 0, (hipStream_t)stream, p);
  return hipGetLastError() == hipSuccess ? SYMPH_OK : SYMPH_ELAUNCH;
}

}  // extern "C"
