// What surrounds the attention of a speculative decoding step: block tables and slot maps from lengths, ancestor masks of
// the drafted trees, the accepted path, and its K,V rows into the paged cache.  The first three are a handful of dependent
// trips to memory per session (their bytes take less than a launch does up to some thousand sessions); the last one, and
// tables for whole arriving sessions, write HBM.
#include "attn_lanes.h"

#include <algorithm>

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
constexpr int kTabStep = kTabThreads * 2;  // tokens of a workgroup whose threads have one pair each
constexpr int kTabPairs = 4;               // pairs of a thread in calls of many tokens,
constexpr int64_t kTabMany = 3 << 18;      // that is
constexpr int64_t kTabMost = (int64_t)(0xFFFFFFFFu / kTabThreads - 1) * kTabStep * kTabPairs;  // (a grid has less than 2^32 threads)

// Sums over the lanes up to this one.  The terms are below 2^37, so the low 24 bits and the rest add up in 32 bits each.
__device__ __forceinline__ int64_t wave_scan64(int64_t v) {
  const unsigned low = wave_inclusive_scan((unsigned)v & 0xFFFFFFu), high = wave_inclusive_scan((unsigned)(v >> 24));
  return ((int64_t)high << 24) + low;
}
__device__ __forceinline__ int32_t clamp32(int64_t v) { return (int32_t)min(max(v, -(int64_t)0x80000000LL), (int64_t)0x7FFFFFFF); }

// Every workgroup owns a run of consecutive new tokens and adds up the lengths of the sessions itself, up to the one its
// tokens end in (64-bit sums: nothing has to be handed over, one launch).  A table entry is written by the thread that has
// the first token of its block.  One more workgroup writes what there is per session.
// A thread has PAIRS pairs of consecutive tokens, kTabStep apart: a pair is one 16-byte store of slots, and the pairs' searches
// and loads wait together.  What bounds it: the chain of lengths, sums, search, free list and store, 5 us with nothing beside
// it (64 sessions, 2200 tokens); 256 arriving sessions of 2.3 million tokens, 28 MB, take 12 us with four pairs a thread, 14
// with two or eight, 20 with one.  One pair fills more of the chip: half a million tokens in 6.5 us against 7.4, a million in
// 10.5 against 8.7, even at three quarters.
template <int PAIRS>
__global__ __launch_bounds__(kTabThreads) void build_tables_kernel(const TablesParams p) {
  __shared__ int32_t first_tok[kTabChunk + 1];  // relative to the run's first token (what does not fit is far from it)
  __shared__ int32_t first_blk[kTabChunk];      // place in the free list
  __shared__ int32_t prefix[kTabChunk], held[kTabChunk];
  __shared__ int64_t wave_sums[kTabThreads / 64][2];
  __shared__ int32_t session_of[2];             // of the run's first token and its last
  constexpr int kRun = kTabStep * PAIRS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool per_session = blockIdx.x == gridDim.x - 1;
  const int64_t t_begin = (int64_t)blockIdx.x * kRun;
  const int run = (int)min((int64_t)kRun, p.total - t_begin);
  const unsigned bs = (unsigned)p.block_size;
  auto block_of = [&](unsigned pos) { return p.bs_shift >= 0 ? pos >> p.bs_shift : pos / bs; };
  auto blocks_for = [&](unsigned n) { return n == 0 ? 0u : block_of(n - 1) + 1; };
  const bool slots16 = ((uintptr_t)p.slot_map & 15) == 0, pos8 = ((uintptr_t)p.positions & 7) == 0;
  typedef long long i64x2 __attribute__((ext_vector_type(2)));
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  auto put = [&](int t, const int64_t* slot, const int32_t* pos, unsigned which) {  // of tokens t (bit 0) and t + 1 (bit 1)
    if (p.slot_map) {
      int64_t* const to = p.slot_map + t_begin + t;
      if (which == 3 && slots16)
        *reinterpret_cast<i64x2*>(to) = i64x2{slot[0], slot[1]};
      else {
        if (which & 1) to[0] = slot[0];
        if (which & 2) to[1] = slot[1];
      }
    }
    if (p.positions) {
      int32_t* const to = p.positions + t_begin + t;
      if (which == 3 && pos8)
        *reinterpret_cast<i32x2*>(to) = i32x2{pos[0], pos[1]};
      else {
        if (which & 1) to[0] = pos[0];
        if (which & 2) to[1] = pos[1];
      }
    }
  };

  int64_t run_tok = 0, run_blk = p.free_begin ? (int64_t)p.free_begin[0] : 0;
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
    int64_t tok_at = run_tok + tok_incl - tok, blk_at = run_blk + blk_incl - blk, chunk_tok = 0, chunk_blk = 0;
#pragma unroll
    for (int w = 0; w < kTabThreads / 64; ++w) {
      if (w < wave) {
        tok_at += wave_sums[w][0];
        blk_at += wave_sums[w][1];
      }
      chunk_tok += wave_sums[w][0];
      chunk_blk += wave_sums[w][1];
    }
    const int chunk_end = clamp32(run_tok + chunk_tok - t_begin);
    const int begin = max(clamp32(run_tok - t_begin), 0), end = min(run, chunk_end);  // the chunk's part of the run
#pragma unroll
    for (int k = 0; k < kTabSess; ++k) {
      const int at = tid * kTabSess + k, i = c0 + at;
      first_tok[at] = clamp32(tok_at - t_begin);
      first_blk[at] = clamp32(blk_at);
      prefix[at] = (int32_t)P[k];
      held[at] = (int32_t)H[k];
      if (per_session && i < p.n_sessions) {
        if (p.cu_new_lens) p.cu_new_lens[i] = (int32_t)tok_at;
        if (p.token_offsets) p.token_offsets[i] = tok_at;
        if (p.held_after) p.held_after[i] = (int32_t)(H[k] + need[k]);
      }
      const int64_t from = tok_at - t_begin, to = from + N[k];
      if (from <= begin && begin < to) session_of[0] = at;
      if (from < end && end <= to) session_of[1] = at;
      tok_at += N[k];
      blk_at += need[k];
    }
    run_tok += chunk_tok;
    run_blk += chunk_blk;
    if (tid == kTabThreads - 1) first_tok[kTabChunk] = chunk_end;
    __syncthreads();
    if (!per_session && begin < end) {
      // The last session that begins at or before a token (those without tokens begin where the next one does)
      const int s0 = session_of[0], range = session_of[1] - s0;
      int t[PAIRS * 2], s[PAIRS * 2];
#pragma unroll
      for (int k = 0; k < PAIRS * 2; ++k) {
        t[k] = (k >> 1) * kTabStep + tid * 2 + (k & 1);
        s[k] = s0;
      }
      for (int step = range > 0 ? 1 << (31 - __builtin_clz(range)) : 0; step > 0; step >>= 1) {
#pragma unroll
        for (int k = 0; k < PAIRS * 2; ++k) {
          const int at = min(s[k] + step, s0 + range);
          if (first_tok[at] <= t[k]) s[k] = at;
        }
      }
      int32_t id[PAIRS * 2], pos[PAIRS * 2], place[PAIRS * 2];
#pragma unroll
      for (int k = 0; k < PAIRS * 2; ++k) {
        const bool in = t[k] >= begin && t[k] < end;
        const unsigned at = (unsigned)prefix[s[k]] + (unsigned)(t[k] - first_tok[s[k]]), b = block_of(at);
        pos[k] = (int32_t)at;
        place[k] = (int32_t)(at - b * bs);
        int32_t* const entry = p.table + (int64_t)(c0 + s[k]) * p.table_stride + b;
        const bool fits = in && b < (unsigned)p.table_stride, taken = b >= (unsigned)held[s[k]];
        const int64_t j = (int64_t)first_blk[s[k]] + (b - (unsigned)held[s[k]]);
        id[k] = -1;
        if (fits && (!taken || (j >= 0 && j < p.n_free))) id[k] = *(taken ? p.free_blocks + j : entry);
        if (fits && taken && place[k] == 0) *entry = id[k];
      }
#pragma unroll
      for (int k = 0; k < PAIRS * 2; k += 2) {
        int64_t slot[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
          slot[u] = id[k + u] >= 0 && id[k + u] < p.n_blocks ? (int64_t)id[k + u] * bs + place[k + u] : -1;
        put(t[k], slot, pos + k, (t[k] >= begin && t[k] < end) | (t[k] + 1 >= begin && t[k] + 1 < end) << 1);
      }
    }
    if (!per_session && chunk_end >= run) return;
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
  // Tokens behind the last session's
  const int64_t none[2] = {-1, -1};
  const int32_t nowhere[2] = {-1, -1};
  const int from = clamp32(run_tok - t_begin);
  for (int t = tid * 2; t < run; t += kTabStep) put(t, none, nowhere, (t >= from) | (t + 1 >= from && t + 1 < run) << 1);
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

constexpr int kMaskTile = 8;               // words of a row that are staged at a time
constexpr int kMaskPitch = kMaskTile + 1;  // (odd: lanes that write the same word of 64 rows meet in no bank)

// A session's nodes in chunks of 64, a node per lane.  Inside a chunk the ancestors follow from six rounds of pointer
// doubling between lanes; the ancestor with the lowest index leads out of the chunk through its parent (a parent comes
// before its children).  What a row has in earlier chunks is then found by one walk over chunks, not over ancestors.
// A row's words go to memory through LDS, so that a wave writes whole lines.  What bounds it: two trips to memory, the rounds
// and the walk, one after another: 3 us for 64 trees of up to 64 nodes, 6.7 for 48 of up to 1001 (3.4 MB of masks).  A call
// of the latter among others takes 6.5, with twice as many threads (fewer chunks looked at twice) 6.9, with half as many 8.2.
__global__ __launch_bounds__(256) void tree_mask_kernel(const TreeMaskParams p) {
  extern __shared__ __attribute__((aligned(16))) char tree_lds[];
  const int cap = (p.max_new + 63) & ~63;
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
  uint64_t* const in_chunk = reinterpret_cast<uint64_t*>(tree_lds);      // ancestors (and self) inside the node's chunk
  uint64_t* const stage = in_chunk + cap + wave * (64 * kMaskPitch);     // of the wave's 64 rows
  int16_t* const way_out = reinterpret_cast<int16_t*>(in_chunk + cap + waves * (64 * kMaskPitch));  // first ancestor before the chunk, -1: none
  const int cu = max(p.cu_new_lens[s], 0);
  const int n = min(min(p.cu_new_lens[s + 1], p.total) - cu, p.max_new);
  const int row0 = blockIdx.y * blockDim.x;
  if (row0 >= n) return;
  const int row_end = min(n, row0 + (int)blockDim.x);
  constexpr int kAhead = 4;  // chunks of a wave whose parents are on their way together
  for (int c0 = wave; c0 * 64 < row_end; c0 += waves * kAhead) {
    int par[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = (c0 + u * waves) * 64 + lane;
      par[u] = i < row_end ? p.parents[cu + i] : -1;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int first = (c0 + u * waves) * 64, i = first + lane;
      if (first >= row_end) break;
      int up = par[u];
      if (up < 0 || up >= i) up = -1;
      int jump = up >= first ? up - first : -1;
      unsigned long long bits = 1ull << lane;
#pragma unroll
      for (int r = 0; r < 6; ++r) {
        const int from = jump < 0 ? lane : jump;
        bits |= __shfl(bits, from);
        const int next = __shfl(jump, from);
        if (jump >= 0) jump = next;
      }
      in_chunk[i] = bits;
      way_out[i] = (int16_t)__shfl(up, __builtin_ctzll(bits));
    }
  }
  __syncthreads();
  const int first = row0 + wave * 64, i = first + lane, rows = min(row_end - first, 64);
  if (rows <= 0) return;
  uint64_t* const to = p.mask + (int64_t)(cu + first) * p.words;
  int x = i < row_end ? i : -1, seen = 0;
  for (int w1 = p.words; w1 > 0; w1 -= kMaskTile) {
    const int w0 = max(w1 - kMaskTile, 0), width = w1 - w0;
    for (int w = width - 1; w >= 0; --w) {
      uint64_t bits = 0;
      if (x >= 0 && (x >> 6) == w0 + w) {
        bits = in_chunk[x];
        x = way_out[x];
        seen += __popcll(bits);
      }
      stage[lane * kMaskPitch + w] = bits;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int lanes = width > 4 ? 8 : width > 2 ? 4 : width;  // per row
    for (int r = lane / lanes; r < rows; r += 64 / lanes) {
      const int w = lane & (lanes - 1);
      if (w < width) to[(int64_t)r * p.words + w0 + w] = stage[r * kMaskPitch + w];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  if (p.positions && i < row_end) p.positions[cu + i] = (p.prefix_lens ? p.prefix_lens[s] : 0) + seen - 1;
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
// enough.  Bound by its trips to memory: 2 us for one tree, 2.3 to 3.7 for 64.
__global__ __launch_bounds__(256) void tree_accept_kernel(const AcceptParams p) {
  const int lane = threadIdx.x & 63;
  const int s = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (s >= p.n_sessions) return;
  const int cu = max(p.cu_new_lens[s], 0);
  const int n = max(min(p.cu_new_lens[s + 1], p.total) - cu, 0);
  const int P = p.prefix_lens ? p.prefix_lens[s] : 0;
  int node = 0, count = n > 0 ? 1 : 0, token = -1;  // the path's last node, its length, the model's token behind it
  for (int c = 0; c < n; c += 64) {
    const int i = c + lane;
    int par = i < n ? p.parents[cu + i] : -1;
    const int drafted = i < n ? p.draft[cu + i] : 0, answer = i < n ? p.target[cu + i] : 0;
    if (par < 0 || par >= i) par = -1;
    // (a parent in the chunk is asked by its lane: one trip to memory less)
    const int near = __shfl(answer, par - c);
    const int wanted = par >= c || par < 0 ? near : p.target[cu + par];
    const bool agrees = par >= 0 && drafted == wanted;
    int mine = i == 0 && n > 0 ? 0 : -1;  // this node's place on the path
    for (;;) {
      const uint64_t next = __ballot(agrees && par == node && i > node);
      if (next == 0) break;
      const int at = __builtin_ctzll(next);
      node = c + at;
      if (lane == at) mine = count;
      ++count;
    }
    if (node >= c) token = __builtin_amdgcn_readlane(answer, node - c);
    if (mine >= 0) p.rows[cu + mine] = cu + i;
  }
  for (int k = count + lane; k < n; k += 64) p.rows[cu + k] = -1;
  if (lane == 0) {
    p.n_accepted[s] = count;
    p.next_tokens[s] = token;
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

// A workgroup has 64 entries of one layer.  Most of them are skipped (a tree has many nodes and one path), so those that are
// written move to the first lanes, and the waves take their rows in turn, K and V as a row each: four rows of a wave at a time,
// whose loads are all on their way before the first store.  The stores stay out of the caches: what the next step reads is spread
// over all heads and layers, and 304 rows of 32 layers (80 MB read and written) took 18.5 us with ordinary stores and 15.6 with
// these (loads that stay out as well: 19.6).  A row's 2 KB are found all over the cache; a large copy moves as much in 12 us.
template <typename VecT>
__global__ __launch_bounds__(256) void kv_commit_kernel(const CommitParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
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
  const uint64_t below = (1ull << lane) - 1;
  const int units = __popcll(valid) * 2;
  const int rank = row >= 0 ? __popcll(valid & below) : units / 2 + __popcll(~valid & below);
  row = __builtin_amdgcn_ds_permute(rank * 4, row);
  const int low = __builtin_amdgcn_ds_permute(rank * 4, (int)dst), high = __builtin_amdgcn_ds_permute(rank * 4, (int)(dst >> 32));
  const int64_t layer_b = (int64_t)blockIdx.y * p.layer_stride_b, new_b = (int64_t)blockIdx.y * p.new_layer_b;
  constexpr int kRows = 4;
  for (int u0 = wave; u0 < units; u0 += 4 * kRows) {
    const VecT* from[kRows];
    VecT* into[kRows];
#pragma unroll
    for (int u = 0; u < kRows; ++u) {
      const int unit = min(u0 + 4 * u, units - 1), at = unit >> 1;
      const int64_t to = (int64_t)__builtin_amdgcn_readlane(high, at) << 32 | (uint32_t)__builtin_amdgcn_readlane(low, at);
      from[u] = reinterpret_cast<const VecT*>((unit & 1 ? p.v_new : p.k_new) + new_b +
                                              (int64_t)__builtin_amdgcn_readlane(row, at) * p.row_bytes);
      into[u] = reinterpret_cast<VecT*>((unit & 1 ? p.v_base : p.k_base) + layer_b + to);
    }
    for (int v = lane; v < p.vecs_per_row; v += 128) {
      const bool two = v + 64 < p.vecs_per_row;
      VecT x[kRows][2];
#pragma unroll
      for (int u = 0; u < kRows; ++u)
        if (u0 + 4 * u < units) {
          x[u][0] = from[u][v];
          if (two) x[u][1] = from[u][v + 64];
        }
#pragma unroll
      for (int u = 0; u < kRows; ++u)
        if (u0 + 4 * u < units) {
          __builtin_nontemporal_store(x[u][0], into[u] + v);
          if (two) __builtin_nontemporal_store(x[u][1], into[u] + v + 64);
        }
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
  if (total_new_tokens > kTabMost) return SYMPH_EUNSUPPORTED;
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
  const bool many = total_new_tokens >= kTabMany;
  const int64_t groups = ceil_div64(total_new_tokens, kTabStep * (many ? kTabPairs : 1)) + 1;
  if (many)
    hipLaunchKernelGGL(build_tables_kernel<kTabPairs>, dim3((unsigned)groups), dim3(kTabThreads), 0, (hipStream_t)stream, p);
  else
    hipLaunchKernelGGL(build_tables_kernel<1>, dim3((unsigned)groups), dim3(kTabThreads), 0, (hipStream_t)stream, p);
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
  if (!grid_takes(n_sessions, threads)) return SYMPH_EUNSUPPORTED;
  const unsigned lds = (unsigned)((max_new_len + 63) & ~63) * 10 + threads * kMaskPitch * 8;
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
  const int64_t groups = ceil_div64(n_sessions, 4);
  if (!grid_takes(groups, 256)) return SYMPH_EUNSUPPORTED;
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
  hipLaunchKernelGGL(tree_accept_kernel, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, p);
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
  const int64_t groups = ceil_div64(n_entries, 64);
  if (row_bytes > 0x7FFFFFFF || cache->n_layers > 65535 || !grid_takes(groups, 256)) return SYMPH_EUNSUPPORTED;
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
  const dim3 grid((unsigned)groups, (unsigned)cache->n_layers);
  if (vec == 16)
    hipLaunchKernelGGL(kv_commit_kernel<u32x4>, grid, dim3(256), 0, (hipStream_t)stream, p);
  else
    hipLaunchKernelGGL(kv_commit_kernel<unsigned int>, grid, dim3(256), 0, (hipStream_t)stream, p);
  return hipGetLastError() == hipSuccess ? SYMPH_OK : SYMPH_ELAUNCH;
}

}  // extern "C"
