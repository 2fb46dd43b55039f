// Blocks that rows of a table share: rows that continue other rows (fork), copies of blocks, references given back and the list
// of free blocks, and the moves that empty a pool's end.  Beside the copies these are a few trips to memory one after another
// over tables and counts of some megabytes at most; the copies are bound by HBM.
#include "attn_lanes.h"

#include <algorithm>

namespace symph {

static int shift_of(int64_t x) { return (x & (x - 1)) == 0 ? __builtin_ctzll((unsigned long long)x) : -1; }

// ---- a row's blocks ----------------------------------------------------------------------------------------------
// Of a row of `len` tokens: blocks that are full, blocks in use, blocks it holds.  A row's blocks end with its table row.
struct RowBlocks {
  int whole, used, held;
};
struct RowShape {
  const int32_t* lens;
  const int32_t* held;
  int32_t stride, block_size, bs_shift;
};
__device__ __forceinline__ RowBlocks blocks_of(const RowShape& s, int len, int held) {
  const unsigned n = (unsigned)max(len, 0);
  const unsigned whole = s.bs_shift >= 0 ? n >> s.bs_shift : n / (unsigned)s.block_size;
  const unsigned used = whole + (whole * (unsigned)s.block_size < n ? 1 : 0), end = (unsigned)s.stride;
  RowBlocks r;
  r.whole = (int)min(whole, end);
  r.used = (int)min(used, end);
  r.held = (int)min(max(used, (unsigned)max(held, 0)), end);
  return r;
}
__device__ __forceinline__ RowBlocks blocks_of_row(const RowShape& s, int row) {
  return blocks_of(s, s.lens[row], s.held ? s.held[row] : 0);
}

// Entry i of n > 0 entries, `none` behind them: asked for unconditionally, so that a thread's loads wait together
__device__ __forceinline__ int entry_or(const int32_t* list, int64_t i, int64_t n, int none) {
  const int v = list[min(i, n - 1)];
  return i < n ? v : none;
}

constexpr int kThreads = 256;

// Sum over a workgroup's threads (every thread gets it); `at`: four words of LDS that no one else is using.
__device__ __forceinline__ int group_sum(int v, int* at) {
  const int incl = wave_inclusive_scan(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) at[threadIdx.x >> 6] = incl;
  __syncthreads();
  return at[0] + at[1] + at[2] + at[3];
}
// Sum over the threads before this one, and of all of them.
__device__ __forceinline__ int group_before(int v, int* at, int* total) {
  const int incl = wave_inclusive_scan(v), wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) at[wave] = incl;
  __syncthreads();
  int before = incl - v;
#pragma unroll
  for (int w = 0; w < 3; ++w)
    if (w < wave) before += at[w];
  *total = at[0] + at[1] + at[2] + at[3];
  return before;
}

// ---- fork --------------------------------------------------------------------------------------------------------
struct ForkParams {
  RowShape shape;
  const int32_t* parents;
  const int32_t* table;
  const int32_t* refs;
  const int32_t* free_blocks;
  const int32_t* free_begin;
  int32_t* table_out;
  int32_t* lens_out;
  int32_t* held_out;
  int32_t* refs_after;
  int32_t* copy_src;
  int32_t* copy_dst;
  int32_t* copy_tokens;
  int32_t* blocks_taken;
  int32_t n_out, n_rows, n_free, n_blocks;
};

// Small calls take one launch, which is what they cost: up to so many table entries, rows (what the LDS arrays hold; a free of 2048 rows
// of 8 entries 10.8 us so, 11.5 in three launches) and, in one workgroup, blocks.  A fork of 8 rows of 507 entries 8.8 us, in two
// launches 10.8; of 16 such rows 12.7 and 10.0.  A free in a pool of 8192 blocks, in one launch and in three: 4096 entries 7.0 and 11.4 us,
// 16384 8.5 and 11.6, 32768 11.5 and 11.8, 65536 17.2 and 14.0; in a pool of 16384 blocks (arrays of twice the size) 14.4 and 11.5.
// A compaction's workgroup goes over its arrays more often, and entries and blocks count together: 2048 blocks and 16384 entries 8.7 us
// and in three launches 10.4; 4096 blocks and 12288 entries 9.6 and 10.4, 16384 10.7 and 10.5; 8192 blocks and 4096 entries 10.3 and
// 11.8, 8192 11.6 and 12.1, 16384 14.1 and 12.2.
constexpr int kFewEntries = 16384, kFewForked = 4096, kFewRows = 1024, kFewBlocks = 8192, kFewMoved = 24 * 1024;
static bool few(int32_t n_rows, int32_t table_stride, int32_t entries = kFewEntries) {
  return n_rows <= kFewRows && (int64_t)n_rows * table_stride <= entries;
}
static bool few_to_compact(int32_t n_rows, int32_t table_stride, int32_t n_blocks) {
  return n_blocks <= kFewBlocks && few(n_rows, table_stride) && n_rows * table_stride + 2 * n_blocks <= kFewMoved;
}
constexpr int kSlice = 4096;  // blocks whose counts a workgroup of a small fork has

// The counts of a slice of the pool after a small fork, every change looked for in the whole table.
__device__ __forceinline__ void fork_slice(const ForkParams& p, int slice, int* lds) {
  __shared__ int change[kSlice], children[kFewRows], whole[kFewRows], held[kFewRows];
  const int tid = threadIdx.x, lo = slice * kSlice, n = min(p.n_blocks - lo, kSlice);
  for (int b = tid; b < kSlice; b += kThreads) change[b] = 0;
  for (int r = tid; r < p.n_rows; r += kThreads) {
    const RowBlocks b = blocks_of_row(p.shape, r);
    children[r] = 0;
    whole[r] = b.whole;
    held[r] = b.held | (b.whole < b.used ? 1 << 30 : 0);  // (bit 30: the last block in use is not full; a row has fewer blocks)
  }
  __syncthreads();
  for (int i = tid; i < p.n_out; i += kThreads) {
    const int up = p.parents[i];
    if (up >= 0 && up < p.n_rows) atomicAdd(children + up, 1);
  }
  __syncthreads();
  int made = 0;
  for (int r = tid; r < p.n_rows; r += kThreads)
    if (held[r] >> 30) made += max(children[r] - 1, 0);
  made = group_sum(made, lds);
  const int entries = p.n_rows * p.shape.stride;
  constexpr int kAhead = 4;
  for (int e0 = tid; e0 < entries; e0 += kThreads * kAhead) {
    int id[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) id[u] = entry_or(p.table, e0 + u * kThreads, entries, -1);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int at = id[u] - lo;
      if (id[u] < 0 || at < 0 || at >= n) continue;
      const int r = (e0 + u * kThreads) / p.shape.stride, c = e0 + u * kThreads - r * p.shape.stride;
      const int more = c < whole[r] ? children[r] - 1 : c < (held[r] & 0x3FFFFFFF) && children[r] == 0 ? -1 : 0;
      if (more != 0) atomicAdd(change + at, more);
    }
  }
  const int64_t begin = p.free_begin ? p.free_begin[0] : 0;
  for (int k = tid; k < made; k += kThreads) {
    const int at = begin + k >= 0 && begin + k < p.n_free ? p.free_blocks[begin + k] - lo : -1;
    if (at >= 0 && at < n) atomicAdd(change + at, 1);
  }
  __syncthreads();
  for (int b = tid; b < n; b += kThreads) p.refs_after[lo + b] = p.refs[lo + b] + change[b];
}

// A workgroup per row of the result, and more that carry the counts over.  A row's place in the free list is the number of rows
// before it that take a block, which every workgroup counts for itself: `first` [n_rows] holds each row's first child.  (512 rows of up
// to 537 entries: 4.6 us, three trips to memory; the launch behind it, atomics on the shared blocks' counts, 6.8.)
template <bool FEW>
__global__ __launch_bounds__(kThreads) void fork_rows_kernel(const ForkParams p) {
  extern __shared__ int fork_lds[];
  int* const first = fork_lds + 4;
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= p.n_out) {
    if (FEW) {
      fork_slice(p, blockIdx.x - p.n_out, fork_lds);
      if (p.n_out == 0 && (int)blockIdx.x == 0 && tid == 0 && p.blocks_taken) p.blocks_taken[0] = p.free_begin ? p.free_begin[0] : 0;
      return;
    }
    const int64_t step = (int64_t)(gridDim.x - p.n_out) * kThreads;
    for (int64_t b = (int64_t)(blockIdx.x - p.n_out) * kThreads + tid; b < p.n_blocks; b += step) p.refs_after[b] = p.refs[b];
    if ((int)blockIdx.x > p.n_out || p.n_out > 0) return;
    if (tid == 0 && p.blocks_taken) p.blocks_taken[0] = p.free_begin ? p.free_begin[0] : 0;
    return;
  }
  const int row = blockIdx.x;
  const bool last = row == p.n_out - 1;
  // What the row itself needs is on its way while the others are counted
  const int up = p.parents[row];
  const bool valid = up >= 0 && up < p.n_rows;
  const int len = valid ? p.shape.lens[up] : 0;
  const RowBlocks b = blocks_of(p.shape, len, valid && p.shape.held ? p.shape.held[up] : 0);
  const int64_t begin = p.free_begin ? p.free_begin[0] : 0;
  const int32_t* const from = p.table + (int64_t)(valid ? up : 0) * p.shape.stride;
  int32_t* const to = p.table_out + (int64_t)row * p.shape.stride;
  constexpr int kAhead = 2;
  int ids[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) ids[u] = valid && p.shape.stride > 0 ? entry_or(from, tid + u * kThreads, p.shape.stride, -1) : -1;

  for (int i = tid; i < p.n_rows; i += kThreads) first[i] = 0x7FFFFFFF;
  __syncthreads();
  for (int i = tid; i <= row; i += kThreads) {
    const int other = p.parents[i];
    if (other >= 0 && other < p.n_rows) atomicMin(first + other, i);
  }
  __syncthreads();
  int before = 0;
  for (int i = tid; i < row; i += kThreads) {
    const int other = p.parents[i];
    if (other < 0 || other >= p.n_rows || first[other] == i) continue;
    const RowBlocks o = blocks_of_row(p.shape, other);
    before += o.whole < o.used;
  }
  before = group_sum(before, fork_lds);
  const bool keeps = valid && first[up] == row, copies = valid && !keeps && b.whole < b.used;
  const int held = !valid ? 0 : keeps ? b.held : b.used;
  const int64_t place = begin + before;
  int made = -1;
  if (copies && place >= 0 && place < p.n_free) made = p.free_blocks[place];
  if (made < 0 || made >= p.n_blocks) made = -1;
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int c = tid + u * kThreads;
    if (c < held) to[c] = copies && c == b.whole ? made : ids[u];
  }
  for (int c = tid + kAhead * kThreads; c < held; c += kThreads) to[c] = copies && c == b.whole ? made : from[c];
  if (tid == 0) {
    p.lens_out[row] = max(len, 0);
    if (p.held_out) p.held_out[row] = held;
    const int src = made >= 0 ? from[b.whole] : -1;
    const bool pair = src >= 0 && src < p.n_blocks;
    p.copy_src[row] = pair ? src : -1;
    p.copy_dst[row] = made;
    p.copy_tokens[row] = made >= 0 ? len - b.whole * p.shape.block_size : 0;
    if (last && p.blocks_taken)
      p.blocks_taken[0] = (int32_t)min(max(place + (copies ? 1 : 0), -(int64_t)0x80000000LL), (int64_t)0x7FFFFFFF);
  }
}

// A workgroup per row of the old table: with c children its full blocks have c - 1 holders more, and what else it holds goes to
// its first child, or to nobody.  One more workgroup counts the new blocks.  (Whole numbers: the order of the additions is free.)
__global__ __launch_bounds__(kThreads) void fork_refs_kernel(const ForkParams p) {
  __shared__ int sums[4];
  const int row = blockIdx.x, tid = threadIdx.x;
  if (row == p.n_rows) {
    for (int i = tid; i < p.n_out; i += kThreads) {
      const int made = p.copy_dst[i];
      if (made >= 0) atomicAdd(p.refs_after + made, 1);
    }
    return;
  }
  const RowBlocks b = blocks_of_row(p.shape, row);
  const int32_t* const from = p.table + (int64_t)row * p.shape.stride;
  constexpr int kAhead = 2;  // entries that are on their way while the children are counted
  int ids[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) ids[u] = p.shape.stride > 0 ? entry_or(from, tid + u * kThreads, p.shape.stride, -1) : -1;
  int children = 0;
  for (int i0 = tid; i0 < p.n_out; i0 += 4 * kThreads)
#pragma unroll
    for (int u = 0; u < 4; ++u) children += entry_or(p.parents, i0 + u * kThreads, p.n_out, -1) == row;
  children = group_sum(children, sums);
  if (children == 1) return;
  const int end = children == 0 ? b.held : b.whole;
  auto add = [&](int c, int id) {
    if (c < end && id >= 0 && id < p.n_blocks) atomicAdd(p.refs_after + id, children - 1);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) add(tid + u * kThreads, ids[u]);
  for (int c = tid + kAhead * kThreads; c < end; c += kThreads) add(c, from[c]);
}

// ---- copies of blocks --------------------------------------------------------------------------------------------
struct CopyParams {
  char* k_base;
  char* v_base;
  const int32_t* src;
  const int32_t* dst;
  const int32_t* tokens;
  int64_t layer_stride_b, block_stride_b;
  int32_t vecs_per_row, block_size, n_blocks, n_pairs;
};

// A workgroup has K or V of one pair in one layer: a contiguous piece, all of it on its way before the first store for blocks of up to
// 32 KB.  Pairs follow each other fastest, so that what runs at a time lies in few pages.  Bound by HBM: 448 blocks of all layers of the
// 8B shape, 1.88 GB read and written, take 343 us (5.5 TB/s; a copy of the same bytes that lie in a row takes 281), with 256 threads
// the same, waves that have such a piece each 372, workgroups that go from piece to piece with the next one's loads under way 356.
constexpr int kCopyThreads = 512;
constexpr int64_t kDenseMost = 1 << 17;  // workgroups
template <typename VecT>
__global__ __launch_bounds__(kCopyThreads) void copy_blocks_kernel(const CopyParams p) {
  const int i = blockIdx.x >> 1, tid = threadIdx.x;
  const int src = p.src[i], dst = p.dst[i], n = p.tokens ? min(max(p.tokens[i], 0), p.block_size) : p.block_size;
  if (src < 0 || src >= p.n_blocks || dst < 0 || dst >= p.n_blocks || src == dst) return;
  char* const base = (blockIdx.x & 1 ? p.v_base : p.k_base) + (int64_t)blockIdx.y * p.layer_stride_b;
  const VecT* const from = reinterpret_cast<const VecT*>(base + (int64_t)src * p.block_stride_b);
  VecT* const to = reinterpret_cast<VecT*>(base + (int64_t)dst * p.block_stride_b);
  const int64_t vecs = (int64_t)n * p.vecs_per_row;
  constexpr int kAhead = 4;
  for (int64_t v = tid; v < vecs; v += kCopyThreads * kAhead) {
    VecT x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (v + kCopyThreads * u < vecs) x[u] = __builtin_nontemporal_load(from + v + kCopyThreads * u);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (v + kCopyThreads * u < vecs) __builtin_nontemporal_store(x[u], to + v + kCopyThreads * u);
  }
}

// The same for long lists, which have few pairs in them as a rule (the moves of a compaction, in room for all there could be; 100 in
// 4096 entries: 90 us, workgroups for every entry 113; 100 in 65536: 141 against 1762; but 1000 in 4096: 833 against 786): a workgroup has 64 pairs of one layer, or a share of them (blockIdx.z).  The pairs that are there move to the first lanes (a
// step of beam search leaves many rows without one) and the waves take their K and V in turn, as a contiguous piece each.
template <typename VecT>
__global__ __launch_bounds__(kThreads) void copy_sparse_kernel(const CopyParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  // (turned from layer to layer: workgroups of the same group would meet on one part of the chip)
  const int i = (int)((blockIdx.x + blockIdx.y + blockIdx.z) % gridDim.x) * 64 + lane;
  int src = -1, dst = -1, n = 0;
  if (i < p.n_pairs) {
    src = p.src[i];
    dst = p.dst[i];
    n = p.tokens ? min(max(p.tokens[i], 0), p.block_size) : p.block_size;
  }
  const bool valid = src >= 0 && src < p.n_blocks && dst >= 0 && dst < p.n_blocks && src != dst && n > 0;
  const uint64_t there = __ballot(valid), below = (1ull << lane) - 1;
  const int pairs = __popcll(there);
  const int rank = valid ? __popcll(there & below) : pairs + __popcll(~there & below);
  src = __builtin_amdgcn_ds_permute(rank * 4, src);
  dst = __builtin_amdgcn_ds_permute(rank * 4, dst);
  n = __builtin_amdgcn_ds_permute(rank * 4, n);
  const int64_t layer_b = (int64_t)blockIdx.y * p.layer_stride_b;
  for (int unit = blockIdx.z * 4 + wave; unit < pairs * 2; unit += gridDim.z * 4) {
    const int at = unit >> 1;
    char* const base = (unit & 1 ? p.v_base : p.k_base) + layer_b;
    const VecT* const from = reinterpret_cast<const VecT*>(base + (int64_t)__builtin_amdgcn_readlane(src, at) * p.block_stride_b);
    VecT* const to = reinterpret_cast<VecT*>(base + (int64_t)__builtin_amdgcn_readlane(dst, at) * p.block_stride_b);
    const int64_t vecs = (int64_t)__builtin_amdgcn_readlane(n, at) * p.vecs_per_row;
    constexpr int kAhead = 8;
    for (int64_t v = lane; v < vecs; v += 64 * kAhead) {
      VecT x[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (v + 64 * u < vecs) x[u] = __builtin_nontemporal_load(from + v + 64 * u);
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (v + 64 * u < vecs) __builtin_nontemporal_store(x[u], to + v + 64 * u);
    }
  }
}

// ---- free blocks and moves ---------------------------------------------------------------------------------------
// The pool's counts in tiles of 1024, so many of them to a workgroup that there are no more workgroups than kMostGroups: each adds
// up what the ones before it counted.
constexpr int kEach = 4, kTile = kThreads * kEach, kMostGroups = 2048;
struct PoolCut {
  int32_t tiles, groups;  // tiles of a workgroup, workgroups
};
static PoolCut cut_pool(int32_t n_blocks) {
  const int64_t tiles = ceil_div64(n_blocks, kTile);
  PoolCut c;
  c.tiles = (int32_t)ceil_div64(tiles, kMostGroups);
  c.groups = (int32_t)ceil_div64(tiles, c.tiles);
  return c;
}
static int64_t round256(int64_t n) { return (n + 255) & ~(int64_t)255; }

struct FreeParams {
  RowShape shape;
  const int32_t* drop;
  const int32_t* taken;  // a list, of which entries *taken_begin .. *taken_end - 1 were taken since the counts
  const int32_t* taken_begin;
  const int32_t* taken_end;
  const int32_t* table;
  const int32_t* refs;
  int32_t* refs_after;
  int32_t* free_blocks;
  int32_t* n_free;
  int32_t* lens_after;
  int32_t* held_after;
  int32_t* counts;  // of every run of 2^run_shift blocks: those that nobody holds
  int32_t n_rows, n_blocks, n_taken, run_shift, n_runs;
};

// Counts are kept for runs of 64 blocks, longer ones where there would be more than kMostGroups: rows that are dropped together change
// them all over, and few counters would make them wait for each other (150 rows with 80000 blocks: 28 us; runs of 1024: 130).
static int run_shift_of(int32_t n_blocks) {
  int s = 6;
  while (((int64_t)kMostGroups << s) < n_blocks) ++s;
  return s;
}

// A wave per run
__global__ __launch_bounds__(kThreads) void free_carry_kernel(const FreeParams p) {
  const int lane = threadIdx.x & 63, run = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (run >= p.n_runs) return;
  int unused = 0;
  for (int64_t i = lane; i < 1ll << p.run_shift; i += 64) {
    const int64_t b = ((int64_t)run << p.run_shift) + i;
    const int r = entry_or(p.refs, b, p.n_blocks, 1);
    if (b < p.n_blocks) p.refs_after[b] = r;
    unused += __popcll(__ballot(r <= 0));
  }
  if (lane == 0) p.counts[run] = unused;
}

// The part of the list that was taken
__device__ __forceinline__ void taken_range(const FreeParams& p, int* begin, int* end) {
  *begin = *end = 0;
  if (!p.taken) return;
  *end = min(p.taken_end[0], p.n_taken);
  *begin = min(max(p.taken_begin ? p.taken_begin[0] : 0, 0), max(*end, 0));
}

// A workgroup per row, and one for the blocks that were taken.  (A quarter of 512 rows dropped, a pool of 131072: the carry 2.6 us,
// this 4.2, the list behind it 3.7; with the unused blocks counted in the last launch instead of here the call took 18, now 11.6.)  (A count that passes from 0 to 1 or back, in whatever order the changes
// come, ends where the run's count of unused blocks says.)
__global__ __launch_bounds__(kThreads) void free_rows_kernel(const FreeParams p) {
  const int row = blockIdx.x, tid = threadIdx.x;
  if (row == p.n_rows) {
    int begin, end;
    taken_range(p, &begin, &end);
    for (int64_t i = begin + tid; i < end; i += kThreads) {
      const int id = p.taken[i];
      if (id < 0 || id >= p.n_blocks) continue;
      if (atomicAdd(p.refs_after + id, 1) == 0) atomicSub(p.counts + (id >> p.run_shift), 1);
    }
    return;
  }
  const int len = p.shape.lens[row];
  const RowBlocks b = blocks_of(p.shape, len, p.shape.held ? p.shape.held[row] : 0);
  const bool gone = p.drop[row] != 0;
  if (gone) {
    const int32_t* const from = p.table + (int64_t)row * p.shape.stride;
    constexpr int kAhead = 2;
    for (int c0 = tid; c0 < b.held; c0 += kAhead * kThreads) {
      int id[kAhead], were[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) id[u] = entry_or(from, c0 + u * kThreads, b.held, -1);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) were[u] = id[u] >= 0 && id[u] < p.n_blocks ? atomicSub(p.refs_after + id[u], 1) : 0;
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (were[u] == 1) atomicAdd(p.counts + (id[u] >> p.run_shift), 1);
    }
  }
  __syncthreads();  // (the lengths may be written over)
  if (tid == 0) {
    if (p.lens_after) p.lens_after[row] = gone ? 0 : len;
    if (p.held_after) p.held_after[row] = gone ? 0 : b.held;
  }
}

// What the groups before `group`, those before `other`, and all of them counted
struct Counted {
  int before, other, total;
};
__device__ __forceinline__ Counted counted(const int32_t* counts, int groups, int group, int other, int (*at)[3]) {
  int n[kMostGroups / kThreads], sum[3] = {0, 0, 0};
#pragma unroll
  for (int u = 0; u < kMostGroups / kThreads; ++u) n[u] = entry_or(counts, threadIdx.x + u * kThreads, groups, 0);
#pragma unroll
  for (int u = 0; u < kMostGroups / kThreads; ++u) {
    const int g = threadIdx.x + u * kThreads;
    sum[0] += g < group ? n[u] : 0;
    sum[1] += g < other ? n[u] : 0;
    sum[2] += n[u];
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int incl = wave_inclusive_scan(sum[k]);
    if ((threadIdx.x & 63) == 63) at[threadIdx.x >> 6][k] = incl;
  }
  __syncthreads();
  Counted c;
  c.before = at[0][0] + at[1][0] + at[2][0] + at[3][0];
  c.other = at[0][1] + at[1][1] + at[2][1] + at[3][1];
  c.total = at[0][2] + at[1][2] + at[2][2] + at[3][2];
  return c;
}

// A workgroup per kListRuns runs
constexpr int kListRuns = kTile / 64;
__global__ __launch_bounds__(kThreads) void free_list_kernel(const FreeParams p) {
  __shared__ int sums[4], known[4][3];
  const int tiles = 1 << (p.run_shift - 6);
  const int64_t begin = (int64_t)blockIdx.x * tiles * kTile;
  const Counted all = counted(p.counts, p.n_runs, blockIdx.x * kListRuns, 0, known);
  const int total = all.total;
  int at = all.before;
  if (blockIdx.x == 0 && threadIdx.x == 0) p.n_free[0] = total;
  for (int t = 0; t < tiles; ++t) {
    const int64_t b0 = begin + (int64_t)t * kTile + threadIdx.x * kEach;
    int unused[kEach], n = 0;
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      unused[u] = entry_or(p.refs_after, b0 + u, p.n_blocks, 1) <= 0;
      n += unused[u];
    }
    int in_tile;
    int to = at + group_before(n, sums, &in_tile);
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      if (unused[u]) p.free_blocks[to++] = (int32_t)(b0 + u);
      if (b0 + u >= total && b0 + u < p.n_blocks) p.free_blocks[b0 + u] = -1;  // behind the list's end
    }
    at += in_tile;
  }
}

// ---- small pools: one workgroup ----
constexpr int kOne = 1024, kOneEach = kFewBlocks / kOne;  // its threads, consecutive blocks of a thread

// Sum over the threads before this one of a workgroup of kOne, and of all of them
__device__ __forceinline__ int one_before(int v, int* at, int* total) {
  const int incl = wave_inclusive_scan(v), wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) at[wave] = incl;
  __syncthreads();
  int before = incl - v, all = 0;
#pragma unroll
  for (int w = 0; w < kOne / 64; ++w) {
    if (w < wave) before += at[w];
    all += at[w];
  }
  *total = all;
  return before;
}

__global__ __launch_bounds__(kOne) void free_few_kernel(const FreeParams p) {
  __shared__ int refs[kFewBlocks], ends[kFewRows], sums[kOne / 64];
  const int tid = threadIdx.x, entries = p.n_rows * p.shape.stride;
  for (int b = tid; b < p.n_blocks; b += kOne) refs[b] = p.refs[b];
  for (int r = tid; r < p.n_rows; r += kOne) {
    const int len = p.shape.lens[r];
    const RowBlocks b = blocks_of(p.shape, len, p.shape.held ? p.shape.held[r] : 0);
    const bool gone = p.drop[r] != 0;
    ends[r] = gone ? b.held : 0;
    if (p.lens_after) p.lens_after[r] = gone ? 0 : len;
    if (p.held_after) p.held_after[r] = gone ? 0 : b.held;
  }
  __syncthreads();
  for (int e = tid; e < entries; e += kOne) {
    const int r = e / p.shape.stride;
    if (e - r * p.shape.stride >= ends[r]) continue;
    const int id = p.table[e];
    if (id >= 0 && id < p.n_blocks) atomicSub(refs + id, 1);
  }
  int begin, end;
  taken_range(p, &begin, &end);
  for (int64_t i = begin + tid; i < end; i += kOne) {
    const int id = p.taken[i];
    if (id >= 0 && id < p.n_blocks) atomicAdd(refs + id, 1);
  }
  __syncthreads();
  int unused[kOneEach], n = 0;
#pragma unroll
  for (int u = 0; u < kOneEach; ++u) {
    const int b = tid * kOneEach + u;
    unused[u] = b < p.n_blocks && refs[b] <= 0;
    n += unused[u];
  }
  int total;
  int to = one_before(n, sums, &total);
#pragma unroll
  for (int u = 0; u < kOneEach; ++u)
    if (unused[u]) p.free_blocks[to++] = tid * kOneEach + u;
  for (int b = tid; b < p.n_blocks; b += kOne) {
    p.refs_after[b] = refs[b];
    if (b >= total) p.free_blocks[b] = -1;
  }
  if (tid == 0) p.n_free[0] = total;
}

struct CompactParams {
  RowShape shape;
  const int32_t* refs;
  const int32_t* table;
  int32_t* table_out;
  int32_t* refs_after;
  int32_t* map;
  int32_t* src;
  int32_t* dst;
  int32_t* result;  // blocks in use, moves, blocks that stay behind
  int32_t* counts;  // per workgroup: blocks in use
  int32_t* place;   // per block: which move it leaves or is taken by, -1: none
  int32_t n_rows, n_blocks, n_keep, n_pairs, tiles;
};

__global__ __launch_bounds__(kThreads) void compact_count_kernel(const CompactParams p) {
  __shared__ int sums[4];
  const int64_t begin = (int64_t)blockIdx.x * p.tiles * kTile;
  int used = 0;
  for (int t = 0; t < p.tiles; ++t)
#pragma unroll
    for (int u = 0; u < kEach; ++u)
      used += entry_or(p.refs, begin + (int64_t)t * kTile + u * kThreads + threadIdx.x, p.n_blocks, 0) > 0;
  used = group_sum(used, sums);
  if (threadIdx.x == 0) p.counts[blockIdx.x] = used;
}

// Which move a block leaves by, or is taken by
__device__ __forceinline__ void place_block(const CompactParams& p, int b, bool used, int used_before, int keep, int below, int moves) {
  int k = -1;
  if (used && b >= keep) k = used_before - below;
  if (!used && b < keep) k = b - used_before;
  if (k >= moves) k = -1;
  p.place[b] = k;
  if (k >= 0) (used ? p.src : p.dst)[k] = b;
}

// The k-th block in use from `keep` on goes to the k-th block below `keep` that is not.  (A pool of 131072 blocks: the counts 2.3 us, this
// 4.4, the table and the counts afterwards 4.6; each launch is two trips to memory.)
__global__ __launch_bounds__(kThreads) void compact_moves_kernel(const CompactParams p) {
  __shared__ int sums[4], known[4][3], at_edge[4][3];
  const int tid = threadIdx.x;
  // Blocks in use below `keep`: the workgroups' before the one that has it, and that one's own up to it
  const int64_t run = (int64_t)p.tiles * kTile;
  const int edge_known = p.n_keep < 0 ? 0 : (int)(min(p.n_keep, p.n_blocks) / run);
  const Counted all = counted(p.counts, gridDim.x, blockIdx.x, edge_known, known);
  const int total = all.total, keep = p.n_keep < 0 ? total : min(p.n_keep, p.n_blocks);
  const int edge = (int)(keep / run);
  int before = all.before, below = p.n_keep < 0 ? counted(p.counts, gridDim.x, edge, 0, at_edge).before : all.other;
  {
    int n = 0;
    for (int64_t b0 = edge * run + tid; b0 < keep; b0 += kEach * kThreads)
#pragma unroll
      for (int u = 0; u < kEach; ++u) n += entry_or(p.refs, b0 + u * kThreads, keep, 0) > 0;
    below += group_sum(n, sums);
  }
  const int moves = min(min(keep - below, total - below), p.n_pairs);
  if (blockIdx.x == 0 && tid == 0) {
    p.result[0] = total;
    p.result[1] = moves;
    p.result[2] = total - below - moves;
  }
  for (int64_t t = 0; t < p.tiles; ++t) {
    const int64_t b0 = blockIdx.x * run + t * kTile + tid * kEach;
    int used[kEach], n = 0;
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      used[u] = entry_or(p.refs, b0 + u, p.n_blocks, 0) > 0;
      n += used[u];
    }
    int in_tile;
    int used_before = before + group_before(n, sums, &in_tile);
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
      if (b0 + u < p.n_blocks) place_block(p, (int)(b0 + u), used[u], used_before, keep, below, moves);
      used_before += used[u];
    }
    before += in_tile;
  }
  for (int64_t k = moves + (int64_t)blockIdx.x * kThreads + tid; k < p.n_pairs; k += (int64_t)gridDim.x * kThreads) {
    p.src[k] = -1;
    p.dst[k] = -1;
  }
}

// The first workgroups have the table's rows, the others the pool.
__global__ __launch_bounds__(kThreads) void compact_apply_kernel(const CompactParams p) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x < p.n_rows) {
    const int row = blockIdx.x, held = blocks_of_row(p.shape, row).held;
    for (int c = tid; c < held; c += kThreads) {
      const int64_t at = (int64_t)row * p.shape.stride + c;
      int id = p.table[at];
      if (id >= 0 && id < p.n_blocks) {
        const int k = p.place[id];
        if (k >= 0 && p.refs[id] > 0) id = p.dst[k];
      }
      p.table_out[at] = id;
    }
    return;
  }
  const int64_t step = (int64_t)(gridDim.x - p.n_rows) * kThreads;
  for (int64_t b = (int64_t)(blockIdx.x - p.n_rows) * kThreads + tid; b < p.n_blocks; b += step) {
    const int k = p.place[b], refs = p.refs[b];
    const bool leaves = k >= 0 && refs > 0;
    p.map[b] = leaves ? p.dst[k] : (int32_t)b;
    p.refs_after[b] = leaves ? 0 : k >= 0 ? p.refs[p.src[k]] : refs;
  }
}

__global__ __launch_bounds__(kOne) void compact_few_kernel(const CompactParams p) {
  __shared__ uint16_t to[kFewBlocks], src[kFewBlocks / 2], dst[kFewBlocks / 2];  // (there are no more moves than half of the blocks)
  __shared__ int held[kFewRows], sums[kOne / 64];
  const int tid = threadIdx.x, entries = p.n_rows * p.shape.stride;
  for (int r = tid; r < p.n_rows; r += kOne) held[r] = blocks_of_row(p.shape, r).held;
  int refs[kOneEach], n = 0;
#pragma unroll
  for (int u = 0; u < kOneEach; ++u) {
    const int b = tid * kOneEach + u;
    refs[u] = entry_or(p.refs, b, p.n_blocks, 0);
    n += refs[u] > 0;
    to[b] = (uint16_t)b;
  }
  int total;
  const int used_before = one_before(n, sums, &total);
  const int keep = p.n_keep < 0 ? total : min(p.n_keep, p.n_blocks);
  int below = 0;
#pragma unroll
  for (int u = 0; u < kOneEach; ++u) below += refs[u] > 0 && tid * kOneEach + u < keep;
  int all_below;
  one_before(below, sums, &all_below);
  const int moves = min(min(keep - all_below, total - all_below), p.n_pairs);
  int used = used_before;
#pragma unroll
  for (int u = 0; u < kOneEach; ++u) {
    const int b = tid * kOneEach + u;
    if (b >= p.n_blocks) break;
    const int k = refs[u] > 0 ? (b >= keep ? used - all_below : moves) : (b < keep ? b - used : moves);
    used += refs[u] > 0;
    if (k >= moves)
      p.refs_after[b] = refs[u];
    else if (refs[u] > 0)
      src[k] = (uint16_t)b;
    else
      dst[k] = (uint16_t)b;
  }
  __syncthreads();
  for (int k = tid; k < p.n_pairs; k += kOne) {
    const bool there = k < moves;
    const int from = there ? src[k] : -1, into = there ? dst[k] : -1;
    p.src[k] = from;
    p.dst[k] = into;
    if (there) {
      to[from] = (uint16_t)into;
      p.refs_after[into] = p.refs[from];
      p.refs_after[from] = 0;
    }
  }
  __syncthreads();
  for (int b = tid; b < p.n_blocks; b += kOne) p.map[b] = to[b];
  for (int e = tid; e < entries; e += kOne) {
    const int r = e / p.shape.stride;
    if (e - r * p.shape.stride >= held[r]) continue;
    const int id = p.table[e];
    p.table_out[e] = id >= 0 && id < p.n_blocks ? to[id] : id;
  }
  if (tid == 0) {
    p.result[0] = total;
    p.result[1] = moves;
    p.result[2] = total - all_below - moves;
  }
}

// Checks that all of these share: a table of rows.  n_rows == 0 needs no arrays.
static int32_t check_rows(const int32_t* d_lens, const int32_t* d_table, int32_t table_stride, int32_t n_rows, int32_t block_size,
                          int32_t n_blocks) {
  if (n_rows < 0 || table_stride < 0 || block_size <= 0 || n_blocks <= 0) return SYMPH_EINVAL;
  if (n_rows > 0 && (!d_lens || (table_stride > 0 && !d_table))) return SYMPH_EINVAL;
  return SYMPH_OK;
}
static RowShape shape_of(const int32_t* d_lens, const int32_t* d_held, int32_t table_stride, int32_t block_size) {
  RowShape s;
  s.lens = d_lens;
  s.held = d_held;
  s.stride = table_stride;
  s.block_size = block_size;
  s.bs_shift = shift_of(block_size);
  return s;
}
static int32_t launched() { return hipGetLastError() == hipSuccess ? SYMPH_OK : SYMPH_ELAUNCH; }

}  // namespace symph

using namespace symph;

extern "C" {

int32_t symph_kv_fork(const int32_t* d_parents, int32_t n_out, const int32_t* d_lens, const int32_t* d_held_blocks, int32_t n_rows,
                      const int32_t* d_block_table, int32_t table_stride, int32_t block_size, int32_t n_blocks,
                      const int32_t* d_refs, const int32_t* d_free_blocks, int32_t n_free, const int32_t* d_free_begin,
                      int32_t* d_table_out, int32_t* d_lens_out, int32_t* d_held_out, int32_t* d_refs_after,
                      int32_t* d_copy_src, int32_t* d_copy_dst, int32_t* d_copy_tokens, int32_t* d_blocks_taken, void* stream) {
  const int32_t rc = check_rows(d_lens, d_block_table, table_stride, n_rows, block_size, n_blocks);
  if (rc != SYMPH_OK) return rc;
  if (n_out < 0 || n_free < 0 || !d_refs || !d_refs_after || (n_free > 0 && !d_free_blocks)) return SYMPH_EINVAL;
  if (n_out > 0 && (!d_parents || !d_lens_out || !d_copy_src || !d_copy_dst || !d_copy_tokens || (table_stride > 0 && !d_table_out)))
    return SYMPH_EINVAL;
  if (d_refs_after == d_refs || (d_blocks_taken && d_blocks_taken == d_free_begin)) return SYMPH_EINVAL;
  if (n_out > 0 && n_rows > 0 &&
      (d_lens_out == d_lens || (d_held_out && d_held_out == d_held_blocks) || (table_stride > 0 && d_table_out == d_block_table)))
    return SYMPH_EINVAL;
  if (n_rows > SYMPH_FORK_MAX_ROWS || n_out > SYMPH_FORK_MAX_ROWS) return SYMPH_EUNSUPPORTED;
  ForkParams p;
  p.shape = shape_of(d_lens, d_held_blocks, table_stride, block_size);
  p.parents = d_parents;
  p.table = d_block_table;
  p.refs = d_refs;
  p.free_blocks = d_free_blocks;
  p.free_begin = d_free_begin;
  p.table_out = d_table_out;
  p.lens_out = d_lens_out;
  p.held_out = d_held_out;
  p.refs_after = d_refs_after;
  p.copy_src = d_copy_src;
  p.copy_dst = d_copy_dst;
  p.copy_tokens = d_copy_tokens;
  p.blocks_taken = d_blocks_taken;
  p.n_out = n_out;
  p.n_rows = n_rows;
  p.n_free = n_free;
  p.n_blocks = n_blocks;
  const unsigned lds = (4 + n_rows) * 4;
  if (few(n_rows, table_stride, kFewForked) && n_out <= kFewRows) {
    hipLaunchKernelGGL(fork_rows_kernel<true>, dim3((unsigned)(n_out + ceil_div64(n_blocks, kSlice))), dim3(kThreads), lds,
                       (hipStream_t)stream, p);
    return launched();
  }
  const int64_t carry = std::min<int64_t>(ceil_div64(n_blocks, kTile), kMostGroups);
  hipLaunchKernelGGL(fork_rows_kernel<false>, dim3((unsigned)(n_out + carry)), dim3(kThreads), lds, (hipStream_t)stream, p);
  hipLaunchKernelGGL(fork_refs_kernel, dim3((unsigned)n_rows + 1), dim3(kThreads), 0, (hipStream_t)stream, p);
  return launched();
}

int32_t symph_kv_copy_blocks(const symph_kv_cache* cache, const int32_t* d_src_blocks, const int32_t* d_dst_blocks,
                             const int32_t* d_tokens, int32_t n_pairs, void* stream) {
  const int32_t rc = validate_cache(cache);
  if (rc != SYMPH_OK) return rc;
  if (n_pairs < 0) return SYMPH_EINVAL;
  if (n_pairs == 0) return SYMPH_OK;
  if (!d_src_blocks || !d_dst_blocks) return SYMPH_EINVAL;
  const int eb = elem_bytes_of(cache->dtype);
  const int64_t row_bytes = (int64_t)cache->n_kv_heads * cache->head_dim * eb, groups = ceil_div64(n_pairs, 64);
  if (row_bytes > 0x7FFFFFFF || cache->n_layers > 65535 || !grid_takes(groups, kThreads)) return SYMPH_EUNSUPPORTED;
  CopyParams p;
  p.k_base = (char*)cache->k_base;
  p.v_base = (char*)cache->v_base;
  p.src = d_src_blocks;
  p.dst = d_dst_blocks;
  p.tokens = d_tokens;
  p.layer_stride_b = cache->layer_stride * eb;
  p.block_stride_b = cache->block_stride * eb;
  const uintptr_t align_or = (uintptr_t)p.k_base | (uintptr_t)p.v_base | (uintptr_t)p.layer_stride_b | (uintptr_t)p.block_stride_b |
                             (uintptr_t)row_bytes;
  if (align_or & 3) return SYMPH_EUNSUPPORTED;
  const int vec = (align_or & 15) ? 4 : 16;
  p.vecs_per_row = (int32_t)(row_bytes / vec);
  p.block_size = cache->block_size;
  p.n_blocks = cache->n_blocks;
  p.n_pairs = n_pairs;
  if (2 * (int64_t)n_pairs * cache->n_layers <= kDenseMost) {
    const dim3 grid((unsigned)n_pairs * 2, (unsigned)cache->n_layers);
    if (vec == 16)
      hipLaunchKernelGGL(copy_blocks_kernel<u32x4>, grid, dim3(kCopyThreads), 0, (hipStream_t)stream, p);
    else
      hipLaunchKernelGGL(copy_blocks_kernel<unsigned int>, grid, dim3(kCopyThreads), 0, (hipStream_t)stream, p);
  } else {
    const int64_t shares = std::min<int64_t>(32, std::max<int64_t>(1, kDenseMost / (groups * cache->n_layers)));
    const dim3 grid((unsigned)groups, (unsigned)cache->n_layers, (unsigned)shares);
    if (vec == 16)
      hipLaunchKernelGGL(copy_sparse_kernel<u32x4>, grid, dim3(kThreads), 0, (hipStream_t)stream, p);
    else
      hipLaunchKernelGGL(copy_sparse_kernel<unsigned int>, grid, dim3(kThreads), 0, (hipStream_t)stream, p);
  }
  return launched();
}

int64_t symph_kv_free_workspace_bytes(int32_t n_blocks) {
  return n_blocks <= 0 ? SYMPH_EINVAL : round256(ceil_div64(n_blocks, 1ll << run_shift_of(n_blocks)) * 4);
}

int32_t symph_kv_free(const int32_t* d_drop, const int32_t* d_lens, const int32_t* d_held_blocks, int32_t n_rows,
                      const int32_t* d_block_table, int32_t table_stride, int32_t block_size, int32_t n_blocks,
                      const int32_t* d_refs, int32_t* d_refs_after, int32_t* d_free_blocks, int32_t* d_n_free,
                      int32_t* d_lens_after, int32_t* d_held_after, const int32_t* d_taken_blocks, int32_t n_taken,
                      const int32_t* d_taken_begin, const int32_t* d_taken_end, void* d_workspace, int64_t workspace_bytes,
                      void* stream) {
  const int32_t rc = check_rows(d_lens, d_block_table, table_stride, n_rows, block_size, n_blocks);
  if (rc != SYMPH_OK) return rc;
  if (n_taken < 0 || (d_taken_blocks && !d_taken_end) || (d_taken_blocks && d_taken_blocks == d_free_blocks)) return SYMPH_EINVAL;
  if (!d_refs || !d_refs_after || !d_free_blocks || !d_n_free || (n_rows > 0 && !d_drop) || workspace_bytes < 0) return SYMPH_EINVAL;
  if (d_refs_after == d_refs || d_free_blocks == d_refs || d_free_blocks == d_refs_after) return SYMPH_EINVAL;
  if (!grid_takes((int64_t)n_rows + 1, kThreads)) return SYMPH_EUNSUPPORTED;
  if (!d_workspace || workspace_bytes < symph_kv_free_workspace_bytes(n_blocks)) return SYMPH_EWORKSPACE;
  if (((uintptr_t)d_workspace & 255) != 0) return SYMPH_EUNSUPPORTED;
  FreeParams p;
  p.shape = shape_of(d_lens, d_held_blocks, table_stride, block_size);
  p.drop = d_drop;
  p.taken = n_taken > 0 ? d_taken_blocks : nullptr;
  p.taken_begin = d_taken_begin;
  p.taken_end = d_taken_end;
  p.n_taken = n_taken;
  p.table = d_block_table;
  p.refs = d_refs;
  p.refs_after = d_refs_after;
  p.free_blocks = d_free_blocks;
  p.n_free = d_n_free;
  p.lens_after = d_lens_after;
  p.held_after = d_held_after;
  p.counts = (int32_t*)d_workspace;
  p.n_rows = n_rows;
  p.n_blocks = n_blocks;
  p.run_shift = run_shift_of(n_blocks);
  p.n_runs = (int32_t)ceil_div64(n_blocks, 1ll << p.run_shift);
  if (n_blocks <= kFewBlocks && few(n_rows, table_stride)) {
    hipLaunchKernelGGL(free_few_kernel, dim3(1), dim3(kOne), 0, (hipStream_t)stream, p);
    return launched();
  }
  hipLaunchKernelGGL(free_carry_kernel, dim3((unsigned)ceil_div64(p.n_runs, 4)), dim3(kThreads), 0, (hipStream_t)stream, p);
  const unsigned changes = (unsigned)n_rows + (p.taken ? 1 : 0);
  if (changes > 0) hipLaunchKernelGGL(free_rows_kernel, dim3(changes), dim3(kThreads), 0, (hipStream_t)stream, p);
  hipLaunchKernelGGL(free_list_kernel, dim3((unsigned)ceil_div64(p.n_runs, kListRuns)), dim3(kThreads), 0, (hipStream_t)stream, p);
  return launched();
}

int64_t symph_kv_compact_workspace_bytes(int32_t n_blocks) {
  return n_blocks <= 0 ? SYMPH_EINVAL : round256((int64_t)cut_pool(n_blocks).groups * 4) + round256((int64_t)n_blocks * 4);
}

int32_t symph_kv_compact(const int32_t* d_refs, int32_t n_blocks, int32_t n_keep, const int32_t* d_lens,
                         const int32_t* d_held_blocks, int32_t n_rows, const int32_t* d_block_table, int32_t table_stride,
                         int32_t block_size, int32_t* d_table_out, int32_t* d_refs_after, int32_t* d_block_map,
                         int32_t* d_copy_src, int32_t* d_copy_dst, int32_t n_pairs, int32_t* d_counts, void* d_workspace,
                         int64_t workspace_bytes, void* stream) {
  const int32_t rc = check_rows(d_lens, d_block_table, table_stride, n_rows, block_size, n_blocks);
  if (rc != SYMPH_OK) return rc;
  if (!d_refs || !d_refs_after || !d_block_map || !d_counts || n_pairs < 0 || workspace_bytes < 0) return SYMPH_EINVAL;
  if (n_pairs > 0 && (!d_copy_src || !d_copy_dst || d_copy_src == d_copy_dst)) return SYMPH_EINVAL;
  if (n_rows > 0 && table_stride > 0 && !d_table_out) return SYMPH_EINVAL;
  if (d_refs_after == d_refs || d_block_map == d_refs || d_block_map == d_refs_after) return SYMPH_EINVAL;
  const PoolCut cut = cut_pool(n_blocks);
  const int64_t groups = n_rows + (int64_t)std::min<int64_t>(ceil_div64(n_blocks, kTile), kMostGroups);
  if (!grid_takes(groups, kThreads)) return SYMPH_EUNSUPPORTED;
  if (!d_workspace || workspace_bytes < symph_kv_compact_workspace_bytes(n_blocks)) return SYMPH_EWORKSPACE;
  if (((uintptr_t)d_workspace & 255) != 0) return SYMPH_EUNSUPPORTED;
  CompactParams p;
  p.shape = shape_of(d_lens, d_held_blocks, table_stride, block_size);
  p.refs = d_refs;
  p.table = d_block_table;
  p.table_out = d_table_out;
  p.refs_after = d_refs_after;
  p.map = d_block_map;
  p.src = d_copy_src;
  p.dst = d_copy_dst;
  p.result = d_counts;
  p.counts = (int32_t*)d_workspace;
  p.place = (int32_t*)((char*)d_workspace + round256((int64_t)cut.groups * 4));
  p.n_rows = n_rows;
  p.n_blocks = n_blocks;
  p.n_keep = n_keep;
  p.n_pairs = n_pairs;
  p.tiles = cut.tiles;
  if (few_to_compact(n_rows, table_stride, n_blocks)) {
    hipLaunchKernelGGL(compact_few_kernel, dim3(1), dim3(kOne), 0, (hipStream_t)stream, p);
    return launched();
  }
  hipLaunchKernelGGL(compact_count_kernel, dim3(cut.groups), dim3(kThreads), 0, (hipStream_t)stream, p);
  hipLaunchKernelGGL(compact_moves_kernel, dim3(cut.groups), dim3(kThreads), 0, (hipStream_t)stream, p);
  hipLaunchKernelGGL(compact_apply_kernel, dim3((unsigned)groups), dim3(kThreads), 0, (hipStream_t)stream, p);
  return launched();
}

}  // extern "C"
