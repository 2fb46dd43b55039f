// tree_attn: drafted tokens against [paged cached prefix ; the drafted tokens themselves under a bit mask].
//   x_j = scale q.k_j over the keys j that the row sees, p = softmax(x), out = sum_j p_j v_j; zero for a row that sees nothing.
//
// The N drafted tokens of a session and the G query heads of a kv-head are N * G query rows that read the same keys.  Three
// kernels, by how many rows there are and of what type; in each a workgroup has one kv-head and a tile of rows:
//   wide    bf16, more than 64 rows: tiles of 128 rows, keys through LDS, bound by the matrix cores
//   stream  bf16, up to 64 rows: every wave reads keys of its own, bound by memory
//   fp32    tiles of 16 to 64 rows on the fp32 matrix instruction
// and a wave per row where addresses are not on 16 bytes.  What they share:
//   * Scores are computed transposed, S^T = K Q^T: a query per lane, so the softmax state is a scalar of the lane, and the
//     probabilities a lane holds are the operand of O^T += V^T P^T as they are.
//   * Statistics and sums are fp32.  Probabilities go into the bf16 products as two values, 16 bits in all: rounded to the 8 bits of
//     one they would be as far off as the values of a flat softmax over a few hundred keys cancel.  It costs the wide kernel half
//     again as many products (14 % of its time).
//   * Every key block has one 32-bit word per query row that says which of its keys the row sees: all ones inside the prefix,
//     the low bits in its last block, the caller's mask in the blocks of the tree, which start at the tree's first token.
//   * Trees are small and prefixes long: where the tiles do not fill the chip the key axis is cut, the parts leave (maximum, sum,
//     unnormalised rows) in the workspace and a second launch joins them.  Every workgroup works out its part from the lengths.
#include "attn_lanes.h"

#include <algorithm>
#include <type_traits>

namespace symph {

struct TreeParams {
  const void* k_layer;
  const void* v_layer;
  int64_t block_stride;  // elements
  int32_t n_blocks, block_size, n_kv_heads, n_q_heads;
  const void* q;
  const void* k_new;
  const void* v_new;
  void* out;
  const uint32_t* mask;
  int32_t mask_words;  // 32-bit words of a row
  const int32_t* cu_new_lens;
  const int32_t* prefix_lens;
  const int32_t* table;
  int32_t table_stride, n_sessions, total;
  float scale;
  uint32_t group_bytes;  // bytes between blocks where the rows of a load lie in one block and a block fits 32 bits; else 0
  uint32_t bs_magic, bs_more;  // key / block_size = key * bs_magic >> 32 >> bs_more for keys below 2^31, block_size > 1
  int32_t max_pieces;    // of tiles (per kv-head) or ranges: what the grid and the workspace have room for
  int32_t c_min;         // key blocks of a tile that are not cut further, of a range at least
  int32_t cut;           // 0: one piece per tile
  int32_t aligned;       // narrow tiles: cut into pieces, not ranges
  int32_t slots;         // workgroups per kv-head that are on the chip at once
  int32_t group, group_shift, heads_shift;  // query heads of a kv-head; log2 of it and of n_kv_heads, or -1
  float* parts;
};

static __device__ __attribute__((aligned(256))) const unsigned kNoRow[128] = {};  // a head's row of zeros

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__bf16 x) { return (float)x; }

// Scores are kept in units of the exponential that the type uses: base 2 in bf16, e in fp32.
template <typename T>
__device__ __forceinline__ float exp_of(float x) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(x);
  return expf(x);
}
template <typename T>
__device__ __forceinline__ float score_scale(float scale) {
  return sizeof(T) == 2 ? scale * 1.4426950408889634f : scale;
}

// A score, or minus infinity where bit `at` of `seen` is clear: two bit operations (written as a choice it became a branch per
// score, 26 000 lines of them).
__device__ __forceinline__ float score_if(uint32_t seen, int at, float x) {
  const unsigned keep = (unsigned)((int)(seen << (31 - at)) >> 31);
  return __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, x) & keep) | (0xFF800000u & ~keep));
}

// ---- which piece of which tile a workgroup has --------------------------------------------------------------------
struct TreePiece {
  int s, cu, P, N;
  int tile, index, count;  // tile of the session, piece of the tile, pieces of each of its tiles
  int block0, block1;      // key blocks: the prefix's first, then the tree's
  int stride;              // between the numbers of a tile's consecutive pieces
};

template <int BM, int KB>
__device__ __forceinline__ void tree_session(const TreeParams& p, int G, int i, int& cu, int& P, int& N, int& tiles,
                                             int& blocks) {
  cu = P = N = tiles = blocks = 0;
  if (i >= p.n_sessions) return;
  cu = max(p.cu_new_lens[i], 0);
  N = max(min(p.cu_new_lens[i + 1], p.total) - cu, 0);
  P = max(p.prefix_lens[i], 0);
  if (N == 0) return;
  tiles = (N * G + BM - 1) / BM;
  blocks = P / KB + (P % KB != 0) + (N + KB - 1) / KB;
}

// A session's key blocks times tiles, as a lane's share of a 64-lane sum of 32 bits.  (The host refuses calls whose bounds allow a
// session more than that: 10^9 keys.)
constexpr int kMostWork = 0x7FFFFFFF / 64;
__device__ __forceinline__ int share_of_work(int tiles, int blocks) { return (int)min((int64_t)tiles * blocks, (int64_t)kMostWork); }

// (Divisions are forty instructions, and a call of one session is short: shifts where there is a power of two.)
__device__ __forceinline__ int token_of(const TreeParams& p, unsigned row) {
  return (int)(p.group_shift >= 0 ? row >> p.group_shift : row / (unsigned)p.group);
}
__device__ __forceinline__ void split_block(const TreeParams& p, unsigned block, int& kvh, int& rest) {
  rest = (int)(p.heads_shift >= 0 ? block >> p.heads_shift : block / (unsigned)p.n_kv_heads);
  kvh = (int)block - rest * p.n_kv_heads;
}

constexpr int kPieceCost = 8;  // start, end and join of a piece of a wide tile, in blocks of 64 keys

// Piece `g` of the batch.  A tile of b key blocks is cut into ceil(b / c) near-equal pieces, of a length c that depends on the whole
// batch; the tiles of a session have their pieces of the same keys beside each other.  Every wave works
// this out by itself, a session per lane: no scheduling launch, no barrier.
template <int BM, int KB>
__device__ __forceinline__ bool find_piece(const TreeParams& p, int G, int g, TreePiece& it) {
  const int lane = threadIdx.x & 63;
  int cu, P, N, tiles, blocks;
  int c = 0x7FFFFFFF;
  const bool single = p.n_sessions == 1;  // (then every lane has it: nothing to add up or to search)
  tree_session<BM, KB>(p, G, single ? 0 : lane, cu, P, N, tiles, blocks);
  if (p.cut) {
    int64_t work = share_of_work(tiles, blocks);
    int n_tiles = tiles;
    if (!single) {
      work = __builtin_amdgcn_readlane(wave_inclusive_scan((int)work), 63);
      n_tiles = __builtin_amdgcn_readlane(wave_inclusive_scan(tiles), 63);
    } else {
      work = __builtin_amdgcn_readfirstlane((int)work);
      n_tiles = __builtin_amdgcn_readfirstlane(n_tiles);
    }
    for (int i0 = 64; i0 < p.n_sessions; i0 += 64) {
      int a, b, d, t, k;
      tree_session<BM, KB>(p, G, i0 + lane, a, b, d, t, k);
      work += __builtin_amdgcn_readlane(wave_inclusive_scan(share_of_work(t, k)), 63);
      n_tiles += __builtin_amdgcn_readlane(wave_inclusive_scan(t), 63);
    }
    // Workgroups run in rounds of p.slots per kv-head.  For 1 .. 4 rounds: the length that fills them, half a piece per tile being
    // lost to its last one, and what it takes, rounds times (a piece's blocks and what it costs beside them); the pieces are counted
    // where a lane has all sessions, else bounded.
    if (n_tiles < p.max_pieces && work <= 0x7FFFFFFF) {
      const int least = __builtin_amdgcn_readfirstlane((int)(((unsigned)work + (unsigned)(p.max_pieces - n_tiles) - 1) /
                                                             (unsigned)(p.max_pieces - n_tiles)));
      int best = 0x7FFFFFFF;
#pragma unroll 1
      for (int rounds = 1; rounds <= 4; ++rounds) {
        const int room = p.slots * rounds - (p.aligned ? n_tiles : n_tiles / 2);
        if (room <= 0) continue;
        const int len = max(max(__builtin_amdgcn_readfirstlane((int)(((unsigned)work + (unsigned)room - 1) / (unsigned)room)), least),
                            p.c_min);
        int pieces = tiles * ((blocks + len - 1) / len);
        pieces = single ? __builtin_amdgcn_readfirstlane(pieces)
                 : p.n_sessions <= 64 ? __builtin_amdgcn_readlane(wave_inclusive_scan(pieces), 63)
                                      : p.slots * rounds;
        const int takes = (pieces + p.slots - 1) / p.slots * (len + kPieceCost);
        if (takes < best) {
          best = takes;
          c = len;
        }
        if (len <= p.c_min) break;
      }
      c = __builtin_amdgcn_readfirstlane(c);
    }
  }
  int before = 0;
  for (int i0 = 0; i0 < p.n_sessions; i0 += 64) {
    if (i0 > 0) tree_session<BM, KB>(p, G, i0 + lane, cu, P, N, tiles, blocks);
    const int count = c == 0x7FFFFFFF ? blocks != 0 : (blocks + c - 1) / c, mine = tiles * count;
    const int incl = single ? mine : wave_inclusive_scan(mine);
    const uint64_t holds = __ballot(before + incl > g);
    if (holds) {
      const int at = __builtin_ctzll(holds);
      it.s = i0 + at;
      it.cu = __builtin_amdgcn_readlane(cu, at);
      it.P = __builtin_amdgcn_readlane(P, at);
      it.N = __builtin_amdgcn_readlane(N, at);
      it.count = __builtin_amdgcn_readlane(count, at);
      it.stride = __builtin_amdgcn_readlane(tiles, at);
      const int local = g - before - __builtin_amdgcn_readlane(incl - mine, at), b = __builtin_amdgcn_readlane(blocks, at);
      // (divisions are done on the vector unit: back to scalar registers)
      it.index = it.stride == 1 ? local : __builtin_amdgcn_readfirstlane(local / it.stride);
      it.tile = local - it.index * it.stride;
      const int each = it.count == 1 ? b : __builtin_amdgcn_readfirstlane(b / it.count), longer = b - each * it.count;
      it.block0 = each * it.index + min(it.index, longer);
      it.block1 = it.block0 + each + (it.index < longer);
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// ---- the other way to cut: all tiles' key blocks laid end to end, in session order, and cut into equal ranges, one per workgroup,
// whatever tiles they run through.  Nothing is left over at the end of a launch (pieces of tiles, a third more of them than the
// chip takes at once, made 64 short drafts take 246 us instead of 211); what it costs is that tiles of one session are read at
// different times, so it is for sessions of one tile, and for batches where pieces that end with their tiles would be too unlike
// (see the host's choice).
struct TreeRanges {
  int64_t total, per;  // blocks; of a range
  int count, longer;   // ranges; the first `longer` of them have one block more
  __device__ __forceinline__ int64_t begin(int r) const { return per * r + min(r, longer); }
  __device__ __forceinline__ int holding(int64_t x) const {
    const int64_t head = longer * (per + 1);
    const int64_t a = x < head ? x : x - head, b = x < head ? per + 1 : per;
    const int q = (a | b) >> 31 ? (int)(a / b) : (int)((unsigned)a / (unsigned)b);
    return __builtin_amdgcn_readfirstlane(x < head ? q : longer + q);
  }
};

struct SessionLane {  // what a lane knows of its session
  int cu, P, N, tiles, blocks;
  __device__ __forceinline__ int work() const { return share_of_work(tiles, blocks); }
};

template <int BM, int KB>
__device__ __forceinline__ TreeRanges cut_ranges(const TreeParams& p, int G, SessionLane& mine) {
  const int lane = threadIdx.x & 63;
  const bool single = p.n_sessions == 1;  // (then every lane has it)
  tree_session<BM, KB>(p, G, single ? 0 : lane, mine.cu, mine.P, mine.N, mine.tiles, mine.blocks);
  TreeRanges rg;
  rg.total = single ? __builtin_amdgcn_readfirstlane(mine.work()) : __builtin_amdgcn_readlane(wave_inclusive_scan(mine.work()), 63);
  for (int i0 = 64; i0 < p.n_sessions; i0 += 64) {
    SessionLane other;
    tree_session<BM, KB>(p, G, i0 + lane, other.cu, other.P, other.N, other.tiles, other.blocks);
    rg.total += __builtin_amdgcn_readlane(wave_inclusive_scan(other.work()), 63);
  }
  const int64_t most = rg.total >> 31 ? rg.total / p.c_min : (unsigned)rg.total / (unsigned)p.c_min;
  rg.count = __builtin_amdgcn_readfirstlane((int)max(min(most, (int64_t)p.max_pieces), (int64_t)1));
  rg.per = rg.total >> 31 ? rg.total / rg.count : (unsigned)rg.total / (unsigned)rg.count;
  rg.per = (int64_t)__builtin_amdgcn_readfirstlane((int)(rg.per >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)rg.per);
  rg.longer = (int)(rg.total - rg.per * rg.count);
  return rg;
}

// The tile that block x lies in, all of its blocks; `start`: its first.  mine: the lane's of the first 64 sessions.
template <int BM, int KB>
__device__ __forceinline__ bool find_tile(const TreeParams& p, int G, const SessionLane& mine, int64_t x, TreePiece& it,
                                          int64_t& start) {
  const int lane = threadIdx.x & 63;
  SessionLane here = mine;
  int64_t before = 0;
  for (int i0 = 0; i0 < p.n_sessions; i0 += 64) {
    if (i0 > 0) tree_session<BM, KB>(p, G, i0 + lane, here.cu, here.P, here.N, here.tiles, here.blocks);
    const int work = here.work(), incl = p.n_sessions == 1 ? work : wave_inclusive_scan(work);
    const uint64_t holds = __ballot(before + incl > x);
    if (holds) {
      const int at = __builtin_ctzll(holds);
      it.s = i0 + at;
      it.cu = __builtin_amdgcn_readlane(here.cu, at);
      it.P = __builtin_amdgcn_readlane(here.P, at);
      it.N = __builtin_amdgcn_readlane(here.N, at);
      it.block0 = 0;
      it.block1 = __builtin_amdgcn_readlane(here.blocks, at);
      const int64_t first = before + __builtin_amdgcn_readlane(incl - work, at);
      it.tile = x - first < it.block1 ? 0 : __builtin_amdgcn_readfirstlane((int)(x - first) / it.block1);
      start = first + (int64_t)it.tile * it.block1;
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
  }
  return false;
}

// Results of a cut tile's part in range r: the first place of the range's two if the part starts with the range, else the second.
__device__ __forceinline__ int64_t range_place(const TreeRanges& rg, int r, int64_t tile_start) {
  return 2 * (int64_t)r + (tile_start > rg.begin(r));
}

// A part of a narrow tile in the workspace: its rows, m and l of each, and which part of what it is, for the join (which would
// otherwise work that out again, for 2 us)
struct PartNote {
  int32_t cu, P, N, tile, index, count, own, step;  // count 0: no part.  The tile's first is at place `own`, part c at (own & ~1) + c * step
};
template <int BM, int D>
constexpr int kPartSlot = BM * (D + 2) + (int)(sizeof(PartNote) / 4);
template <int BM, int D>
__device__ __forceinline__ float* part_slot(const TreeParams& p, int64_t place, int kvh) {
  return p.parts + (place * p.n_kv_heads + kvh) * (int64_t)kPartSlot<BM, D>;
}
template <int BM, int D>
__device__ __forceinline__ PartNote* part_note(const TreeParams& p, int64_t place, int kvh) {
  return reinterpret_cast<PartNote*>(part_slot<BM, D>(p, place, kvh) + BM * (D + 2));
}

// Runs `segment(it, place)` for every part of a tile that lies in range r; it.count: 1 if that is all of it, place: else where its
// results go.  Without a cut: for tile r.
template <int BM, int KB, int D, bool PIECES, typename Segment>
__device__ __forceinline__ void for_segments(const TreeParams& p, int G, int kvh, int r, Segment segment) {
  SessionLane mine;
  TreeRanges rg;
  TreePiece it;
  int64_t x = 0, end = 1, start = 0;
  if (p.cut) {
    if (threadIdx.x < 2) *part_note<BM, D>(p, 2 * (int64_t)r + threadIdx.x, kvh) = PartNote{};
    if (!PIECES || !p.aligned) {
      rg = cut_ranges<BM, KB>(p, G, mine);
      if (r >= rg.count) return;
      x = rg.begin(r);
      end = rg.begin(r + 1);
    }
  }
  while (x < end) {
    int64_t place = 0;
    if (!p.cut || (PIECES && p.aligned)) {
      if (!find_piece<BM, KB>(p, G, r, it)) return;
      x = end;
      place = 2 * (int64_t)r;
      if (PIECES && p.cut && threadIdx.x == 0)
        *part_note<BM, D>(p, place, kvh) =
            PartNote{it.cu, it.P, it.N, it.tile, it.index, it.count, 2 * (r - it.index * it.stride), 2 * it.stride};
    } else {
      if (!find_tile<BM, KB>(p, G, mine, x, it, start)) return;
      const int64_t tile_end = start + it.block1, stop = min(tile_end, end);
      it.block0 = (int)(x - start);
      it.block1 = (int)(stop - start);
      it.index = 0;
      it.count = 1;
      if (it.block0 > 0 || stop < tile_end) {
        const int first = rg.holding(start);
        it.index = r - first;
        it.count = rg.holding(tile_end - 1) - first + 1;
        place = range_place(rg, r, start);
        if (threadIdx.x == (place & 1))  // (the thread that has cleared it)
          *part_note<BM, D>(p, place, kvh) =
              PartNote{it.cu, it.P, it.N, it.tile, it.index, it.count, (int)range_place(rg, first, start), 2};
      }
      x = stop;
    }
    if constexpr (PIECES) {
      for (int* v : {&it.s, &it.cu, &it.P, &it.N, &it.tile, &it.count, &it.block0, &it.block1})
        *v = __builtin_amdgcn_readfirstlane(*v);  // (the compiler has them in vector registers)
    }
    segment(it, place);
  }
}

// What a row without any probability gets: zero if it sees no key, NaN if all its scores are minus infinity (0 / 0).
template <typename Piece>
__device__ __forceinline__ float nothing_seen(const TreeParams& p, const Piece& it, int tok) {
  bool sees = it.P > 0;
  const uint32_t* row = p.mask + (int64_t)(it.cu + tok) * p.mask_words;
  for (int w = 0; w < p.mask_words && w * 32 < it.N && !sees; ++w)
    sees = (row[w] & (it.N - w * 32 >= 32 ? ~0u : (1u << (it.N - w * 32)) - 1u)) != 0;
  return sees ? NAN : 0.f;
}

// A row worked out by itself has its probabilities, and with them its sums, 2^24 times smaller than its maximum says: products with
// the largest values a type has then add up without an overflow.
template <typename T>
constexpr float kHeadroom = sizeof(T) == 2 ? 24.0f : 16.635532f;  // log2, or the natural logarithm, of 2^24

// ---- one row by one wave, lanes over the keys of blocks block0 .. block1 - 1, fp32 on the vector unit.  Keys that the row does
// not see are not read.  The result (unnormalised, relative to the maximum m) is left in lds[D .. 2 D - 1]; lds: 2 * D floats of
// the wave's own.  CH columns at a time, the scores worked out again for each.
template <typename T, int D, int KB, int CH>
__device__ __forceinline__ void row_by_lanes(const TreeParams& p, const TreePiece& it, int tok, int h, float* lds, float& m_row,
                                             float& l_row) {
  const int lane = threadIdx.x & 63;
  const int g = token_of(p, (unsigned)h);  // (the kv-head: the same quotient)
  const int prefix_blocks = it.P / KB + (it.P % KB != 0);
  const T* const q = (const T*)p.q + ((int64_t)(it.cu + tok) * p.n_q_heads + h) * D;
  for (int c = lane; c < D; c += 64) lds[c] = widen(q[c]);
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const uint32_t* const mask = p.mask + (int64_t)(it.cu + tok) * p.mask_words;
  const float cs = score_scale<T>(p.scale);
  for (int c0 = 0; c0 < D; c0 += CH) {
    float m = -INFINITY, l = 0.f;
    float acc[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) acc[c] = 0.f;
    for (int64_t v = (int64_t)it.block0 * KB + lane; v < (int64_t)it.block1 * KB; v += 64) {
      const T* kp = nullptr;
      const T* vp = nullptr;
      if (v < (int64_t)prefix_blocks * KB) {
        const int key = (int)v;
        if (key >= it.P) continue;
        const int b = key / p.block_size;
        const int id = b < p.table_stride ? p.table[(int64_t)it.s * p.table_stride + b] : -1;
        if (id >= 0 && id < p.n_blocks) {  // (else a row of zeros: score 0, value 0)
          const int64_t e = (int64_t)id * p.block_stride + ((int64_t)(key - b * p.block_size) * p.n_kv_heads + g) * D;
          kp = (const T*)p.k_layer + e;
          vp = (const T*)p.v_layer + e;
        }
      } else {
        const int j = (int)(v - (int64_t)prefix_blocks * KB);
        if (j >= it.N || (j >> 5) >= p.mask_words || !((mask[j >> 5] >> (j & 31)) & 1)) continue;
        const int64_t e = ((int64_t)(it.cu + j) * p.n_kv_heads + g) * D;
        kp = (const T*)p.k_new + e;
        vp = (const T*)p.v_new + e;
      }
      float dot = 0.f;
      if (kp) {
#pragma unroll 8
        for (int c = 0; c < D; ++c) dot = fmaf(lds[c], widen(kp[c]), dot);
      }
      float x = cs * dot;
      asm("" : "+v"(x));  // (rounded before the maximum is taken off, so that the largest score's exponent is 0 at any size)
      const float m_new = fmaxf(m, x);
      const float ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = exp_of<T>(m - ref);
      const float w = exp_of<T>(x - ref - kHeadroom<T>);
      l = l * alpha + w;
      if (vp) {
#pragma unroll
        for (int c = 0; c < CH; ++c) acc[c] = fmaf(w, widen(vp[c0 + c]), acc[c] * alpha);
      } else {
#pragma unroll
        for (int c = 0; c < CH; ++c) acc[c] *= alpha;
      }
      m = m_new;
    }
    float M = m;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    const float f = m == -INFINITY ? (l == l ? 0.f : 1.f) : exp_of<T>(m - M);
    float lt = l * f;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) lt += __shfl_xor(lt, o);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float a = acc[c] * f;
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) a += __shfl_xor(a, o);
      if (lane == 0) lds[D + c0 + c] = a;  // (a store by lane c each would keep CH lane masks in scalar registers)
    }
    m_row = M == -INFINITY ? M : M + kHeadroom<T>;
    l_row = lt;
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Addresses that the tiled kernel cannot load 16 bytes wide from: a wave per (token, head), all keys.
template <typename T, int D>
__global__ __launch_bounds__(64) void tree_row_kernel(const TreeParams p) {
  constexpr int KB = 32;  // (any: all keys are this wave's)
  __shared__ float lds[2 * D];
  const int lane = threadIdx.x;
  const int tok_all = (int)(blockIdx.x / (unsigned)p.n_q_heads), h = (int)(blockIdx.x % (unsigned)p.n_q_heads);
  int lo = 0, hi = p.n_sessions;  // the last session that begins at or before the token
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.cu_new_lens[mid] <= tok_all)
      lo = mid;
    else
      hi = mid;
  }
  TreePiece it;
  int tiles, blocks;
  tree_session<1, KB>(p, 1, lo, it.cu, it.P, it.N, tiles, blocks);
  const int tok = tok_all - it.cu;
  if (tok < 0 || tok >= it.N) return;
  it.s = lo;
  it.block0 = 0;
  it.block1 = blocks;
  float m, l;
  row_by_lanes<T, D, KB, D>(p, it, tok, h, lds, m, l);
  const float none = l == 0.f ? nothing_seen(p, it, tok) : 0.f;
  T* const out = (T*)p.out + ((int64_t)tok_all * p.n_q_heads + h) * D;
  for (int c = lane; c < D; c += 64) out[c] = (T)(l == 0.f ? none : lds[D + c] * (1.0f / l));
}

// The part of a float that a bf16 value holds without rounding, and two such parts as neighbours of an operand
__device__ __forceinline__ float upper_part(float x) {
  return __builtin_bit_cast(float, __builtin_bit_cast(unsigned, x) & 0xFFFF0000u);
}
__device__ __forceinline__ void put_pair(bf16x8& v, int at, float x, float y) {
  u32x4 words = __builtin_bit_cast(u32x4, v);
  words[at >> 1] = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, y), __builtin_bit_cast(unsigned, x), 0x07060302u);
  v = __builtin_bit_cast(bf16x8, words);
}

// ---- results of a tile of BM rows by all WAVES waves of the workgroup.  slot: where the results of a tile that is cut go.  sum_at(t, r, c, M, L):
// four columns of row r from column c on, added up over the waves that share the row, with their maximum
// and sum; t: turn of the thread.  A row with a value that is not finite (an infinity or a NaN among the values, which the matrix
// product spreads to rows that do not see it), or with scores beyond what the loop's arithmetic is made for, is worked out again
// by itself, from its q: it is not written before (out may be q).  lds: 2 * D floats a wave, which may be where sum_at reads;
// bad_rows: a bit per row, zeros.
constexpr float kLargestScore = 0x1p20f;
template <typename T, int D, int BM, int KB, int WAVES, typename Sum>
__device__ __forceinline__ void finish_tile(const TreeParams& p, const TreePiece& it, float* slot, int kvh, int n_rows, float* lds,
                                            unsigned* bad_rows, Sum sum_at) {
  constexpr int kQuads = BM * D / 4, kTurns = (kQuads + 64 * WAVES - 1) / (64 * WAVES);
  typedef T vec __attribute__((ext_vector_type(4)));
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // (a number that the optimiser cannot see through: no addresses for what follows held in loops before)
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = p.group;
  const unsigned row0 = (unsigned)it.tile * BM;
  const bool whole = it.count == 1;
  // A value of the thread's turn: final for a whole tile
  auto value_of = [&](int t, int r, int c0, float& M, float& L) {
    f32x4 sum = sum_at(t, r, c0, M, L);
    if (L == 0.f) sum = f32x4{0.f, 0.f, 0.f, 0.f};  // (no probability: whatever values the product brought in are not the row's)
    if (whole) {
      if (L == 0.f) {
        const float none = nothing_seen(p, it, token_of(p, row0 + r));
        sum = f32x4{none, none, none, none};
      } else {
        sum *= 1.0f / L;
      }
    }
    return sum;
  };
  // (twice: the values are read from LDS again rather than kept, up to 96 registers)
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int i = tid + t * 64 * WAVES, r = i / (D / 4), c0 = 4 * (i % (D / 4));
    if (i >= kQuads || r >= n_rows) continue;
    float M, L;
    const f32x4 x = value_of(t, r, c0, M, L);
    bool bad = false;
#pragma unroll
    for (int v = 0; v < 4; ++v) bad = bad || !(fabsf(x[v]) < INFINITY);
    // (a sum that is NaN comes from a score that is: every value of the row is NaN either way; so is 0 / 0)
    bad = (bad && L == L && L != 0.f) || (fabsf(M) > kLargestScore && M != -INFINITY);
    if (bad) atomicOr(&bad_rows[r >> 5], 1u << (r & 31));
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int i = tid + t * 64 * WAVES, r = i / (D / 4), c0 = 4 * (i % (D / 4));
    if (i >= kQuads || r >= n_rows || ((bad_rows[r >> 5] >> (r & 31)) & 1)) continue;
    float M, L;
    const f32x4 x = value_of(t, r, c0, M, L);
    if (whole) {
      const unsigned row = row0 + r, tok = (unsigned)token_of(p, row);
      T* const op = (T*)p.out + ((int64_t)(it.cu + (int)tok) * p.n_q_heads + kvh * G + (int)(row - tok * G)) * D;
      vec y;
#pragma unroll
      for (int v = 0; v < 4; ++v) y[v] = (T)x[v];
      *reinterpret_cast<vec*>(op + c0) = y;
    } else {
      *reinterpret_cast<f32x4*>(slot + r * D + c0) = x;
      if (c0 == 0) {
        slot[BM * D + r] = M;
        slot[BM * D + BM + r] = L;
      }
    }
  }
  unsigned any = 0;
#pragma unroll
  for (int word = 0; word < (BM + 31) / 32; ++word) any |= bad_rows[word];
  if (__builtin_amdgcn_readfirstlane(any) == 0) return;
  __syncthreads();  // (lds has been read for the last time)
  int turn = 0;
  for (int word = 0; word < (BM + 31) / 32; ++word)
    for (unsigned left = __builtin_amdgcn_readfirstlane(bad_rows[word]); left; left &= left - 1) {
      if (turn++ % WAVES != wave) continue;
      const int r = word * 32 + __builtin_ctz(left);
      const unsigned row = row0 + r, tok = (unsigned)token_of(p, row);
      const int h = kvh * G + (int)(row - tok * G);
      float* const own = lds + wave * 2 * D;
      float m, l;
      row_by_lanes<T, D, KB, 64>(p, it, (int)tok, h, own, m, l);
      if (whole) {
        T* const op = (T*)p.out + ((int64_t)(it.cu + (int)tok) * p.n_q_heads + h) * D;
        const float none = l == 0.f ? nothing_seen(p, it, (int)tok) : 0.f;
        for (int c = lane; c < D; c += 64) op[c] = (T)(l == 0.f ? none : own[D + c] * (1.0f / l));
      } else {
        for (int c = lane; c < D; c += 64) slot[r * D + c] = own[D + c];
        if (lane == 0) {
          slot[BM * D + r] = m;
          slot[BM * D + BM + r] = l;
        }
      }
    }
}

// LDS layout of rows of K or V such that the 16 rows a quarter-wave reads of K, and the 4 rows x 32 bytes that 16 lanes read of V by
// the transposing read, lie in different banks.  One direct load writes 1 KiB, lane l to place 16 * l: which 16 bytes of which row
// it fetches is what the layout chooses.  Two uses: a tile of 64 keys loaded by the four waves of a workgroup, and one of 8 KB
// loaded by a single wave (stream_*).
template <int D>
struct TileLds;
template <>
struct TileLds<128> {  // 1 KiB: four rows, chunk c of row r at place c ^ ((r & 3) << 2); 16 bytes between such groups
  static constexpr int kGroupRows = 4, kGroup = 1024 + 16, kBytes = 16 * kGroup, kLoads = 4;
  static constexpr int kStreamKeys = 32, kStreamBytes = 8 * kGroup;
  static __device__ __forceinline__ int row_of(int load, int wave, int lane) { return 16 * load + 4 * wave + (lane >> 4); }
  static __device__ __forceinline__ int chunk_of(int, int lane) { return (lane & 15) ^ (((lane >> 4) & 3) << 2); }
  static __device__ __forceinline__ int at(int load, int wave) { return (4 * load + wave) * kGroup; }
  static __device__ __forceinline__ int stream_row(int load, int lane) { return 4 * load + (lane >> 4); }
  static __device__ __forceinline__ int place(int r, int c) { return (r >> 2) * kGroup + (r & 3) * 256 + ((c ^ ((r & 3) << 2)) << 4); }
  // Operand of K for 16 columns `st` of the 32-key half `kb`; k_off[i]: place of the lane's chunk in columns 32 i ..
  static __device__ __forceinline__ bf16x8 k_frag(const char* buf, const int (&k_off)[4], int st, int kb) {
    return *reinterpret_cast<const bf16x8*>(buf + k_off[st >> 1] + 32 * (st & 1) + kb * 8 * kGroup);
  }
  // Operand of V for 16 keys g / 4 and 32 columns g % 4; v_off[i]: place for columns 32 i ..
  static __device__ __forceinline__ bf16x8 v_frag(const char* buf, const int (&v_off)[4], int g) {
    const char* const a = buf + v_off[g & 3] + (g >> 2) * 4 * kGroup;
    const s16x4 lo = lds_read_tr16(reinterpret_cast<const __bf16*>(a));
    const s16x4 hi = lds_read_tr16(reinterpret_cast<const __bf16*>(a + kGroup));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};
template <>
struct TileLds<64> {  // 1 KiB: eight rows, chunk c of row r at place c ^ twist(r)
  static constexpr int kGroupRows = 8, kGroup = 1024, kBytes = 8 * kGroup, kLoads = 2;
  static constexpr int kStreamKeys = 64, kStreamBytes = 8 * kGroup;
  static __device__ __forceinline__ int twist(int r) { return (((r >> 1) & 3) << 1) | ((r >> 3) & 1); }
  static __device__ __forceinline__ int row_of(int load, int wave, int lane) { return 32 * load + 8 * wave + (lane >> 3); }
  static __device__ __forceinline__ int chunk_of(int row, int lane) { return (lane & 7) ^ twist(row); }
  static __device__ __forceinline__ int at(int load, int wave) { return (4 * load + wave) * kGroup; }
  static __device__ __forceinline__ int stream_row(int load, int lane) { return 8 * load + (lane >> 3); }
  static __device__ __forceinline__ int place(int r, int c) { return (r >> 3) * kGroup + (r & 7) * 128 + ((c ^ twist(r)) << 4); }
  static __device__ __forceinline__ bf16x8 k_frag(const char* buf, const int (&k_off)[4], int st, int kb) {
    return *reinterpret_cast<const bf16x8*>(buf + k_off[st] + kb * 4 * kGroup);
  }
  // v_off[2 i + h]: place for columns 32 i .. and half h of the lane's 8 keys
  static __device__ __forceinline__ bf16x8 v_frag(const char* buf, const int (&v_off)[4], int g) {
    const s16x4 lo = lds_read_tr16(reinterpret_cast<const __bf16*>(buf + v_off[2 * (g & 1)] + (g >> 1) * 2 * kGroup));
    const s16x4 hi = lds_read_tr16(reinterpret_cast<const __bf16*>(buf + v_off[2 * (g & 1) + 1] + (g >> 1) * 2 * kGroup));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// 16 bytes a lane from memory straight into LDS, from a scalar base and a lane's 32-bit offset; POLICY 2: non-temporal, for rows
// that are read once.  As a buffer load: beside a flat one under way (a pointer per lane, SYMPH_TREE_GLDS16) the compiler waits for
// every LDS read with "none may be left", because flat loads may use LDS, and the reads ahead of their use were ahead of nothing.
template <int POLICY>
__device__ __forceinline__ void load_lds16(const char* base, unsigned off, char* dst) {
  const __amdgpu_buffer_rsrc_t from = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, 0xFFFFFFFFu, 0x00027000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)dst, 16, off, 0, 0, POLICY);
}
#define SYMPH_TREE_GLDS16(src, dst, POLICY)                                                      \
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(src),         \
                                   (__attribute__((address_space(3))) void*)(dst), 16, 0, POLICY)

// Behind the LDS reads of a buffer and in front of the loads that fill it again, where no barrier is between them: every read has
// returned.  (Program order is not enough: reads and loads into LDS are two queues, and what orders them for other memory, a use of
// the value read, the compiler may move behind the loads.)
__device__ __forceinline__ void lds_reads_returned() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  asm volatile("" ::: "memory");
}

// Where a key's block is in the table (a division would be forty instructions)
__device__ __forceinline__ unsigned table_place(const TreeParams& p, unsigned key) { return __umulhi(key, p.bs_magic) >> p.bs_more; }
__device__ __forceinline__ int block_of_key(const TreeParams& p, int key) {
  return p.block_size == 1 ? key : (int)table_place(p, (unsigned)key);
}
// Where the rows of a load are in a pool, given the load's first key, its place in the block table (from table_place) and the id
// found there; negative: nowhere.  A load has four or eight consecutive keys, which lie in one block of the cache.
__device__ __forceinline__ int64_t rows_at(const TreeParams& p, unsigned key, unsigned at, int id, unsigned row_bytes) {
  const uint64_t off = (uint64_t)(unsigned)id * p.group_bytes + (key - at * (unsigned)p.block_size) * row_bytes;
  return (unsigned)id < (unsigned)p.n_blocks && at < (unsigned)p.table_stride ? (int64_t)off : -1;
}
__device__ __forceinline__ int64_t lane_value(int64_t x, int lane) {
  return (int64_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, lane);
}

// The keys of 32 that a row sees, a bit each: `left` of them exist, `word`: the row's mask (all ones in the prefix).  The words of a
// block are asked for before the loads of the block: asked for when they are needed they would be the youngest load under way, and
// waiting for them waiting for all.
__device__ __forceinline__ uint32_t seen_keys(int left, uint32_t word) {
  return word & (left >= 32 ? ~0u : left > 0 ? (1u << left) - 1u : 0u);
}
__device__ __forceinline__ uint32_t mask_word(const TreeParams& p, const uint32_t* mask_row, int word) {
  return word < 0 ? ~0u : word < p.mask_words ? mask_row[word] : 0u;
}

// Blocks of KEYS of the tree's keys up to the last that a row of the tile sees: with parents before children a tile has no use for
// what comes after its last token.  (A wave looks at all rows of the tile, eight words of each at a time.)
template <int KEYS>
__device__ __forceinline__ int tree_blocks_seen(const TreeParams& p, int cu, int N, unsigned row0, int n_rows) {
  const int lane = threadIdx.x & 63;
  const int from = token_of(p, row0), to = token_of(p, row0 + (unsigned)n_rows - 1);
#pragma unroll 1
  for (int w1 = min((N + 31) >> 5, p.mask_words); w1 > 0; w1 -= 8) {
    uint32_t seen[8] = {};
    for (int t = from + lane; t <= to; t += 64) {
      const uint32_t* const row = p.mask + (int64_t)(cu + t) * p.mask_words;
#pragma unroll
      for (int k = 0; k < 8; ++k) seen[k] |= row[max(w1 - 1 - k, 0)];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (__any(seen[k] != 0)) return (max(w1 - 1 - k, 0) * 32 + 31) / KEYS + 1;
  }
  return 0;
}

// Probabilities of 32 keys, 2^(x * cs - ref), as two bf16 values each, w = hi + lo with 16 bits in all: the leading 8 bits, then
// those of what is left.  Returns the lane's sum of them.
__device__ __forceinline__ float probabilities(const f32x16& x, float cs, float ref, bf16x8 (&hi)[2], bf16x8 (&lo)[2]) {
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int e = 0; e < 16; e += 2) {
    float w[2], rest[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      w[k] = __builtin_amdgcn_exp2f(fmaf(x[e + k], cs, -ref));
      sum[k] += w[k];
      rest[k] = w[k] - upper_part(w[k]);
    }
    put_pair(hi[e >> 3], e & 7, w[0], w[1]);
    put_pair(lo[e >> 3], e & 7, rest[0], rest[1]);
  }
  return sum[0] + sum[1];
}

// ---- narrow tiles (bf16): W waves, RW side by side on the rows, W / RW on the keys.  Up to 64 rows a read of 16 KB of K and V takes
// longer than all arithmetic on it, so a wave is a stream of its own: tiles of 16 KB through two LDS buffers that no other wave
// touches, no barrier.  The K buffer is filled again as soon as the scores are done, the V buffer as soon as the values are.  Loads
// return in order, so "all but the last eight" is exactly the older of the two, which is all that the program waits for; as built the
// compiler adds a wait for all loads in front of a buffer's reads, since it does not tell the two buffers apart, and what keeps memory
// busy meanwhile is the other waves.
// Bound by memory: 64 sessions with drafts of 2 to 8 tokens and 512 to 8192 cached ones (G 4, 1.13 GB) take 206 us, 5.5 TB/s of the
// 6.5 that a copy reaches; the rest is what a workgroup does around its keys, some 15 us, and 25 more where sessions are ragged.
// Four waves in twice as many workgroups take as long, two or one are slower, and so is a barrier per tile.
template <int D, int RW, int W, bool GROUPED>
__global__ __launch_bounds__(64 * W, 2) void tree_stream_kernel(const TreeParams p) {
  typedef __bf16 T;
  typedef TileLds<D> Lds;
  constexpr int BM = 32 * RW, KW = W / RW, KT = Lds::kStreamKeys, NB = KT / 32, NS = D / 16, NT = D / 32;
  __shared__ __attribute__((aligned(16))) char k_lds[W][Lds::kStreamBytes];
  __shared__ __attribute__((aligned(16))) char v_lds[W][Lds::kStreamBytes];
  __shared__ float wave_m[W][32], wave_l[W][32];
  __shared__ unsigned bad_rows[RW];

  const int Hkv = p.n_kv_heads;
  const int G = p.group;
  int kvh, range;
  split_block(p, blockIdx.x, kvh, range);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW;
  const int n = lane & 31;  // query row of this lane within its wave's; also its row of the K operand
  const int kg = lane >> 5;
  for_segments<BM, KT, D, true>(p, G, kvh, range, [&](const TreePiece& it, const int64_t place) {
  const int cu = it.cu, P = it.P, N = it.N;
  const unsigned row0 = (unsigned)it.tile * BM;
  const int n_rows = (int)min((unsigned)BM, (unsigned)N * (unsigned)G - row0);
  const int prefix_tiles = P / KT + (P % KT != 0), full_tiles = P / KT;
  if (tid < RW) bad_rows[tid] = 0;

  const unsigned my_row = row0 + min(rw * 32 + n, n_rows - 1);
  const int tok = token_of(p, my_row);
  const uint32_t* const mask_row = p.mask + (int64_t)(cu + tok) * p.mask_words;
  bf16x8 q[NS];
  {
    const T* const qp = (const T*)p.q + ((int64_t)(cu + tok) * p.n_q_heads + kvh * G + (int)(my_row - (unsigned)tok * G)) * D;
#pragma unroll
    for (int st = 0; st < NS; ++st) q[st] = *reinterpret_cast<const bf16x8*>(qp + 16 * st + 8 * kg);
  }

  // ---- memory -> LDS.  Block ids one per lane, asked for two tiles ahead: lane i has key i of the tile, or the first key of load
  // i & 7 where a load's rows lie in one block.
  const int32_t* const table_row = p.table + (int64_t)it.s * p.table_stride;
  auto block_of = [&](int key) { return block_of_key(p, key); };
  const int begin = it.block0 + kw;
  const int end = rw * 32 < n_rows ? it.block1 : it.block0;  // (waves without a row have no tiles)
  auto my_key = [&](int tile) { return tile * KT + (GROUPED ? (lane & 7) * Lds::kGroupRows : lane & (KT - 1)); };
  auto ask_ids = [&](int tile) {
    const int key = my_key(tile);
    if (tile >= min(prefix_tiles, end) || key >= P) return -1;
    const int j = GROUPED ? (int)table_place(p, (unsigned)key) : block_of(key);
    return j < p.table_stride ? table_row[j] : -1;
  };
  const unsigned row_bytes = (unsigned)(Hkv * D * (int)sizeof(T));
  const char* const k_pool = reinterpret_cast<const char*>((const T*)p.k_layer + kvh * D);
  const char* const v_pool = reinterpret_cast<const char*>((const T*)p.v_layer + kvh * D);
  const char* const k_fresh = reinterpret_cast<const char*>((const T*)p.k_new + (int64_t)cu * Hkv * D + kvh * D);
  const char* const v_fresh = reinterpret_cast<const char*>((const T*)p.v_new + (int64_t)cu * Hkv * D + kvh * D);
  auto find_rows = [&](int tile, int ids) -> int64_t {
    if constexpr (!GROUPED) return 0;
    const unsigned key = (unsigned)my_key(tile);
    return rows_at(p, key, table_place(p, key), ids, row_bytes);
  };
  constexpr int kSplit = D == 64 ? 2 : 1;  // loads differ in the lane's 16 bytes by this many kinds
  unsigned lane_off[kSplit];
#pragma unroll
  for (int i = 0; i < kSplit; ++i) {
    const int row = Lds::stream_row(i, lane);
    lane_off[i] = (unsigned)(row % Lds::kGroupRows) * row_bytes + (unsigned)Lds::chunk_of(row, lane) * 16u;
  }
  constexpr int kPolicy = RW == 1 ? 2 : 0;  // (one wave reads them, or RW)
  // A tile that lies whole in the prefix.  Rows of an id outside the cache come from the row of zeros.
  auto issue_whole = [&](const char* pool, char* buf, int64_t rows) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t at = lane_value(rows, i);
      load_lds16<kPolicy>(at >= 0 ? pool + at : reinterpret_cast<const char*>(kNoRow),
                          at >= 0 ? lane_off[D == 128 ? 0 : i & 1] : (unsigned)(lane % (D / 8)) * 16u, buf + i * Lds::kGroup);
    }
  };
  // Any other tile
  auto issue_rows = [&](const char* pool, const char* fresh, char* buf, int tile, int ids, int64_t rows) {
    int l = lane;
    asm volatile("" : "+v"(l));  // (its pieces of addresses are worked out here: no registers for them in the loop)
    if constexpr (GROUPED) {
      // the prefix's last, or one of the tree: in place of rows that do not exist the last one that does (no row sees them)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = Lds::stream_row(i, l);
        const char* base = reinterpret_cast<const char*>(kNoRow);
        unsigned off = (unsigned)Lds::chunk_of(row, l) * 16u;
        if (tile < prefix_tiles) {
          const int first = tile * KT + i * Lds::kGroupRows;
          const int64_t at = lane_value(rows, i);
          if (first < P && at >= 0) {
            base = pool + at;
            off += (unsigned)min(row % Lds::kGroupRows, P - 1 - first) * row_bytes;
          }
        } else {
          const int first = (tile - prefix_tiles) * KT;
          base = fresh + (uint64_t)first * row_bytes;
          off += (unsigned)min(row, N - 1 - first) * row_bytes;
        }
        load_lds16<kPolicy>(base, off, buf + i * Lds::kGroup);
      }
    } else {
      // small or odd blocks: an address per lane; rows that do not exist are zeros
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = Lds::stream_row(i, l);
        const unsigned in_row = (unsigned)Lds::chunk_of(row, l) * 16u;
        const int id = __shfl(ids, row);
        const char* src = reinterpret_cast<const char*>(kNoRow) + in_row;
        if (tile < prefix_tiles) {
          const int key = tile * KT + row;
          if (key < P && (unsigned)id < (unsigned)p.n_blocks)
            src = pool + (int64_t)id * p.block_stride * (int64_t)sizeof(T) +
                  (uint64_t)(unsigned)(key - block_of(key) * p.block_size) * row_bytes + in_row;
        } else {
          const int j = (tile - prefix_tiles) * KT + row;
          if (j < N) src = fresh + (uint64_t)j * row_bytes + in_row;
        }
        SYMPH_TREE_GLDS16(src, buf + i * Lds::kGroup, kPolicy);
      }
    }
  };

  // ---- LDS reads, as in tree_wide_kernel
  const int krow = key_of_row(n);
  int k_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_off[i] = Lds::place(krow, D == 128 ? 4 * i + kg : 2 * i + kg);
  const int i16 = lane & 15;
  int v_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int dt = D == 128 ? i : i >> 1, half = D == 128 ? 0 : i & 1;
    const int row = 8 * kg + 4 * half + (i16 >> 2);
    v_off[i] = Lds::place(row, 4 * dt + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) + 8 * (i16 & 1);
  }
  char* const k_buf = k_lds[wave];
  char* const v_buf = v_lds[wave];

  f32x16 o[NT];
#pragma unroll
  for (int dt = 0; dt < NT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  float m = -INFINITY, l = 0.f;  // in log2 units
  const float cs = score_scale<T>(p.scale);

  int ids = ask_ids(begin), ids_next = ask_ids(begin + KW);
  uint32_t words[NB] = {};  // of the mask, for the tile at hand
  auto ask_words = [&](int tile) {
#pragma unroll
    for (int b = 0; b < NB; ++b) words[b] = mask_word(p, mask_row, tile < prefix_tiles ? -1 : (tile - prefix_tiles) * NB + b);
  };
  if (begin < end) ask_words(begin);
  int64_t rows = find_rows(begin, ids);
  // Three copies of the loop's body, by what comes after the tile: one that lies whole in the prefix, any other, none.
  enum { kWhole, kRows, kNone };
  auto use_tile = [&](const int tile, auto next) {
    constexpr int kNext = decltype(next)::value;
    __builtin_amdgcn_s_waitcnt(0x0F70 | 8);  // vmcnt(8): K has landed, V may be on its way
    asm volatile("" ::: "memory");
    f32x16 x[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[b][e] = 0.f;
#pragma unroll
    for (int st = 0; st < NS; ++st)
#pragma unroll
      for (int b = 0; b < NB; ++b)
        x[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(Lds::k_frag(k_buf, k_off, st, b), q[st], x[b], 0, 0, 0);
    asm volatile("" ::: "memory");
    uint32_t seen[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) seen[b] = words[b];
    if constexpr (kNext != kNone) {
      ids = ids_next;
      rows = find_rows(tile + KW, ids);
      ids_next = ask_ids(tile + 2 * KW);
    }
    if constexpr (kNext == kRows) ask_words(tile + KW);
    if constexpr (kNext != kNone) lds_reads_returned();
    if constexpr (kNext == kWhole) issue_whole(k_pool, k_buf, rows);
    if constexpr (kNext == kRows) issue_rows(k_pool, k_fresh, k_buf, tile + KW, ids, rows);
    if (kNext != kWhole && tile >= full_tiles) {
      const int left = tile < prefix_tiles ? P - tile * KT : N - (tile - prefix_tiles) * KT;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const uint32_t bits = seen_keys(left - 32 * b, seen[b]) >> (8 * kg);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[b][e] = score_if(bits, 16 * (e >> 3) + (e & 7), x[b][e]);
      }
    }
    float mx = x[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, x[b][e]);
    const float m_new = fmaxf(m, max_across_halves(mx) * cs);
    if (__any(m_new > m)) {
      const float a = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= a;
#pragma unroll
      for (int dt = 0; dt < NT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= a;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    bf16x8 hi[NB][2], lo[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) l += probabilities(x[b], cs, ref, hi[b], lo[b]);
    if constexpr (kNext != kNone)
      __builtin_amdgcn_s_waitcnt(0x0F70 | 8);  // V has landed, the next K may be on its way
    else
      __builtin_amdgcn_s_waitcnt(0x0F70);
    asm volatile("" ::: "memory");
#pragma unroll
    for (int g = 0; g < 2 * NB * NT; ++g) {
      const int step = g / NT;
      const bf16x8 v = Lds::v_frag(v_buf, v_off, g);
      o[g % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, hi[step >> 1][step & 1], o[g % NT], 0, 0, 0);
      o[g % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, lo[step >> 1][step & 1], o[g % NT], 0, 0, 0);
    }
    if constexpr (kNext != kNone) lds_reads_returned();
    if constexpr (kNext == kWhole) issue_whole(v_pool, v_buf, rows);
    if constexpr (kNext == kRows) issue_rows(v_pool, v_fresh, v_buf, tile + KW, ids, rows);
  };
  if (begin < end) {
    const int whole_end = GROUPED ? min(end, full_tiles) : begin;
    if (GROUPED && begin < whole_end) {
      issue_whole(k_pool, k_buf, rows);
      issue_whole(v_pool, v_buf, rows);
    } else {
      issue_rows(k_pool, k_fresh, k_buf, begin, ids, rows);
      issue_rows(v_pool, v_fresh, v_buf, begin, ids, rows);
    }
    int tile = begin;
    if constexpr (GROUPED) {
      for (; tile + KW < whole_end; tile += KW) use_tile(tile, std::integral_constant<int, kWhole>{});
    }
    for (; tile + KW < end; tile += KW) use_tile(tile, std::integral_constant<int, kRows>{});
    use_tile(tile, std::integral_constant<int, kNone>{});
  }

  // ---- the KW waves of a row group: maximum, factors, and their rows through the wave's own buffers (16 rows in each, 16-byte
  // piece c of row r at c ^ r)
  const float l_row = sum_across_halves(l);
  if (lane < 32) wave_m[wave][n] = m;
  __syncthreads();
  float M = -INFINITY;
#pragma unroll
  for (int w = 0; w < KW; ++w) M = fmaxf(M, wave_m[w * RW + rw][n]);
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
  if (lane < 32) wave_l[wave][n] = m == -INFINITY ? l_row : l_row * f;  // (no maximum: 0, or NaN scores)
  constexpr int kPieces = D / 4;
  auto row_at = [&](int w, int r) { return reinterpret_cast<float*>(r < 16 ? k_lds[w] : v_lds[w]) + (r & 15) * D; };
  if (rw * 32 < n_rows) {
    float* const mine = row_at(wave, n);
#pragma unroll
    for (int dt = 0; dt < NT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(mine + 4 * ((8 * dt + kg + 2 * i) ^ (n & (kPieces - 1)))) =
            f32x4{o[dt][4 * i] * f, o[dt][4 * i + 1] * f, o[dt][4 * i + 2] * f, o[dt][4 * i + 3] * f};
  }
  __syncthreads();
  finish_tile<T, D, BM, KT, W>(p, it, part_slot<BM, D>(p, place, kvh), kvh, n_rows, reinterpret_cast<float*>(k_lds), bad_rows,
                               [&](int, int r, int c0, float& Mr, float& L) {
    const int first = r >> 5, i = r & 31;  // the first of the row's waves
    Mr = -INFINITY;
    L = 0.f;
    f32x4 sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      Mr = fmaxf(Mr, wave_m[first + w * RW][i]);
      L += wave_l[first + w * RW][i];
      sum += *reinterpret_cast<const f32x4*>(row_at(first + w * RW, i) + 4 * ((c0 / 4) ^ (i & (kPieces - 1))));
    }
    return sum;
  });
  __syncthreads();  // (the buffers and flags of this segment are used again)
  });
}

// ---- fp32: W waves, RW side by side on rows (16 each), W / RW on the keys (blocks of 16); the fp32 matrix instruction
// throughout.  K and V go from memory into operand registers (V's operand has one value per lane: no transposing).
// Few rows: bound by memory (41 sessions of 16064 to 31443 keys and up to 3 tokens, 1 GB: 190 us, 5.2 TB/s) or, small, by its trips
// to it: 8 tokens behind 256 take 10.2 us, 5.2 of them three blocks of a wave, 2 in front of the first.  Many rows: by the first
// cache, which every wave reads K and V from for itself (16 KB per 64 products of 128-wide heads): a third to a half of the matrix
// cores' rate.  Two blocks on their way instead of one were slower for small calls (12.2 against 10.7 us), and so were lines of the
// second and third asked for with the first (11.1): a longer program.
constexpr int kFp32Rows = 16;
template <int D, int RW, int W>
__global__ __launch_bounds__(64 * W, 2) void tree_fp32_kernel(const TreeParams p) {
  typedef float T;
  constexpr int R = kFp32Rows, BM = R * RW, KW = W / RW;
  constexpr int kStride = D + 4;  // floats between rows of the results
  __shared__ __attribute__((aligned(16))) char lds[W * R * kStride * 4];
  __shared__ float wave_m[W][R], wave_l[W][R];
  __shared__ unsigned bad_rows[(BM + 31) / 32];

  const int Hkv = p.n_kv_heads;
  const int G = p.group;
  int kvh, range;
  split_block(p, blockIdx.x, kvh, range);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rw = wave % RW, kw = wave / RW;
  const int n = lane & (R - 1);  // query row of this lane within its wave's; also its row of the K operand
  const int kg = lane / R;       // its share of the contraction index: half (bf16) or quarter (fp32) of the wave
  for_segments<BM, R, D, false>(p, G, kvh, range, [&](const TreePiece& it, const int64_t place) {
  const int cu = it.cu, P = it.P, N = it.N;
  const unsigned row0 = (unsigned)it.tile * BM;
  const int n_rows = (int)min((unsigned)BM, (unsigned)N * (unsigned)G - row0);
  const int prefix_blocks = P / R + (P % R != 0);
  if (tid < (BM + 31) / 32) bad_rows[tid] = 0;

  const unsigned my_row = row0 + min(rw * R + n, n_rows - 1);
  const int tok = token_of(p, my_row);
  const T* const qp = (const T*)p.q + ((int64_t)(cu + tok) * p.n_q_heads + kvh * G + (int)(my_row - (unsigned)tok * G)) * D;
  const uint32_t* const mask_row = p.mask + (int64_t)(cu + tok) * p.mask_words;

  auto block_of = [&](int key) { return block_of_key(p, key); };
  const int32_t* const table_row = p.table + (int64_t)it.s * p.table_stride;
  // Block ids one per lane (lane i: key i of the block), passed between lanes
  auto fetch_id = [&](int blk) {
    const int key = blk * R + n;
    if (blk >= min(prefix_blocks, it.block1) || key >= P) return -1;
    const int j = block_of(key);
    return j < p.table_stride ? table_row[j] : -1;
  };
  // Row r of the prefix's key block blk
  auto row_of = [&](const void* pool, int blk, int r, int id) {
    const int key = blk * R + r;
    if (key >= P || id < 0 || id >= p.n_blocks) return (const T*)kNoRow;
    return (const T*)pool + (int64_t)id * p.block_stride + ((int64_t)(key - block_of(key) * p.block_size) * Hkv + kvh) * D;
  };
  // The word of the mask for a block, and the keys of the block that the lane's row sees, a bit each
  auto ask_word = [&](int blk) { return mask_word(p, mask_row, blk < prefix_blocks ? -1 : ((blk - prefix_blocks) * R) >> 5); };
  auto seen_of = [&](int blk, uint32_t word) -> uint32_t {
    if (blk < prefix_blocks) return seen_keys(P - blk * R, word);
    const int at = (blk - prefix_blocks) * R;
    return seen_keys(N - (at & ~31), word) >> (at & 31);
  };
  const unsigned row_bytes = (unsigned)(Hkv * D * (int)sizeof(T));
  auto load_vec = [](const void* at) { return *(const u32x4 __attribute__((address_space(1)))*)(uintptr_t)at; };
  auto load16 = [&](const char* base, unsigned lane_off) {
    if constexpr (D == 128) asm("" : "+s"(base), "+v"(lane_off));
    return load_vec(base + lane_off);
  };
  const char* const k_head = (const char*)((const T*)p.k_layer + kvh * D);
  const char* const v_head = (const char*)((const T*)p.v_layer + kvh * D);
  const char* const k_fresh = (const char*)((const T*)p.k_new + (int64_t)cu * Hkv * D + kvh * D);
  const char* const v_fresh = (const char*)((const T*)p.v_new + (int64_t)cu * Hkv * D + kvh * D);

  const int first = it.block0 + kw;
  const int last = rw * R < n_rows ? it.block1 : it.block0;  // (waves without a row have no blocks)
  const float cs = score_scale<T>(p.scale);
  float m = -INFINITY, l = 0.f;
  float* const mine = reinterpret_cast<float*>(lds) + (rw * KW + kw) * R * kStride;  // the wave's part of the results

  // Between the loop and the results: the row's maximum over the KW waves, this wave's factor
  auto share_state = [&](float l_row) {
    if (lane < R) wave_m[rw * KW + kw][n] = m;
    __syncthreads();  // (also: no wave reads its V tile any more, the buffer is free)
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < KW; ++w) M = fmaxf(M, wave_m[rw * KW + w][n]);
    const float f = m == -INFINITY ? 0.f : exp_of<T>(m - M);
    if (lane < R) wave_l[rw * KW + kw][n] = m == -INFINITY ? l_row : l_row * f;  // (no maximum: 0, or NaN scores)
    return f;
  };

  constexpr int NS = D / 16;  // 16-byte loads of a row per lane
  constexpr int NH = D / 64;  // groups of 64 output columns
  f32x4 q[NS];
#pragma unroll
  for (int j = 0; j < NS; ++j) q[j] = *reinterpret_cast<const f32x4*>(qp + 16 * j + 4 * kg);
  f32x4 kr[NS], vr[4][NH];
  const unsigned k_off = n * row_bytes + 16 * kg, v_off_mem = 4 * kg * row_bytes + 16 * n;
  auto load_block = [&](int blk, int id) {
    if (p.group_bytes != 0 || blk >= prefix_blocks) {
      // The rows of eight keys each follow each other: from a scalar address and a lane's constant where the sixteen do, else from
      // two.  In place of rows that do not exist the last one that does (no row sees them), rows of zeros where there is no block.
      const char *k_at[2], *v_at[2];
      unsigned step[2] = {row_bytes, row_bytes};
      int last;
      bool whole = true;
      if (blk >= prefix_blocks) {
        const int j = (blk - prefix_blocks) * 16;
        last = N - 1 - j;
        k_at[0] = k_fresh + (uint64_t)j * row_bytes;
        v_at[0] = v_fresh + (uint64_t)j * row_bytes;
        k_at[1] = k_at[0] + 8 * row_bytes;
        v_at[1] = v_at[0] + 8 * row_bytes;
      } else {
        last = P - 1 - blk * 16;
        int64_t at[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const unsigned key = (unsigned)(blk * 16 + 8 * i);
          at[i] = rows_at(p, key, table_place(p, key), __builtin_amdgcn_readlane(id, 8 * i), row_bytes);
          k_at[i] = at[i] < 0 ? (const char*)kNoRow : k_head + at[i];
          v_at[i] = at[i] < 0 ? (const char*)kNoRow : v_head + at[i];
          if (at[i] < 0) step[i] = 0;
        }
        whole = at[0] >= 0 && at[1] == at[0] + 8 * (int64_t)row_bytes;
      }
      if (whole && last >= 15) {
#pragma unroll
        for (int j = 0; j < NS; ++j) kr[j] = __builtin_bit_cast(f32x4, load16(k_at[0] + 64 * j, k_off));
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int h = 0; h < NH; ++h)
            vr[e][h] = __builtin_bit_cast(f32x4, load16(v_at[0] + e * row_bytes + 256 * h, v_off_mem));
        return;
      }
      const int kr_row = min(n, last);
      const char* const k_row = (kr_row & 8 ? k_at[1] : k_at[0]) + (kr_row & 7) * (kr_row & 8 ? step[1] : step[0]) + 16 * kg;
#pragma unroll
      for (int j = 0; j < NS; ++j) kr[j] = __builtin_bit_cast(f32x4, load_vec(k_row + 64 * j));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = min(4 * kg + e, last);
        const char* const v_row = (row & 8 ? v_at[1] : v_at[0]) + (row & 7) * (row & 8 ? step[1] : step[0]) + 16 * n;
#pragma unroll
        for (int h = 0; h < NH; ++h) vr[e][h] = __builtin_bit_cast(f32x4, load_vec(v_row + 256 * h));
      }
      return;
    }
    const T* const k_row = row_of(p.k_layer, blk, n, id) + 4 * kg;
#pragma unroll
    for (int j = 0; j < NS; ++j) kr[j] = __builtin_bit_cast(f32x4, load_vec(k_row + 16 * j));
#pragma unroll
    for (int e = 0; e < 4; ++e) {  // key 4 * kg + e: values 64 * h + 4 * n .. + 3 of its row
      const T* const v_row = row_of(p.v_layer, blk, 4 * kg + e, __shfl(id, 4 * kg + e)) + 4 * n;
#pragma unroll
      for (int h = 0; h < NH; ++h) vr[e][h] = __builtin_bit_cast(f32x4, load_vec(v_row + 64 * h));
    }
  };
  // o[h][c][e]: column 64 * h + 16 * kg + 4 * e + c of row n.  A sum over thousands of keys in one chain loses bits: kRun blocks
  // are added up by themselves (o_run, l_run) before they join the rest.
  constexpr int kRun = 8;
  f32x4 o[NH][4], o_run[NH][4];
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int c = 0; c < 4; ++c) o[h][c] = o_run[h][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  float l_run = 0.f;
  auto join_run = [&]() {
    l += l_run;
    l_run = 0.f;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        o[h][c] += o_run[h][c];
        o_run[h][c] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
  };
  int run = 0;
  int id_next = first < last ? fetch_id(first) : -1;
  uint32_t word = first < last ? ask_word(first) : 0u;
  const int id_first = id_next;
  id_next = fetch_id(first + KW);
  if (first < last) load_block(first, id_first);
  for (int blk = first; blk < last; blk += KW) {
    f32x4 sc[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) sc[e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(kr[j][e], q[j][e], sc[e], 0, 0, 0);
    f32x4 v[4][NH];
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int h = 0; h < NH; ++h) v[e][h] = vr[e][h];
    const uint32_t my_word = word;
    const int id = id_next;
    id_next = fetch_id(blk + 2 * KW);
    if (blk + KW < last) {
      word = ask_word(blk + KW);
      load_block(blk + KW, id);
    }
    float x[4];  // key 4 * kg + e
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = cs * ((sc[0][e] + sc[1][e]) + (sc[2][e] + sc[3][e]));
      asm("" : "+v"(x[e]));  // (rounded before the maximum is taken off, so that the largest score's exponent is 0 at any size)
    }
    if (blk >= prefix_blocks || (blk + 1) * 16 > P) {
      const uint32_t bits = seen_of(blk, my_word) >> (4 * kg);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[e] = score_if(bits, e, x[e]);
    }
    float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float m_new = fmaxf(m, mx);
    if (__any(m_new > m)) {
      const float a = m == -INFINITY ? 0.f : expf(m - m_new);
      m = m_new;
      l *= a;
      l_run *= a;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          o[h][c] *= a;
          o_run[h][c] *= a;
        }
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float w = expf(x[e] - ref);
      l_run += w;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          o_run[h][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][h][c], w, o_run[h][c], 0, 0, 0);
    }
    if (++run == kRun) {
      join_run();
      run = 0;
    }
  }
  join_run();
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  const float f = share_state(l);
  if (rw * R < n_rows) {
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4*>(mine + n * kStride + 64 * h + 16 * kg + 4 * e) =
            f32x4{o[h][0][e] * f, o[h][1][e] * f, o[h][2][e] * f, o[h][3][e] * f};
  }
  __syncthreads();

  const float* const all = reinterpret_cast<const float*>(lds);
  finish_tile<T, D, BM, R, W>(p, it, part_slot<BM, D>(p, place, kvh), kvh, n_rows, reinterpret_cast<float*>(lds), bad_rows,
                              [&](int, int r, int c0, float& M, float& L) {
    const int w0 = (r / R) * KW;
    M = -INFINITY;
    L = 0.f;
    f32x4 sum{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      L += wave_l[w0 + w][r % R];
      M = fmaxf(M, wave_m[w0 + w][r % R]);
      sum += *reinterpret_cast<const f32x4*>(all + ((w0 + w) * R + r % R) * kStride + c0);
    }
    return sum;
  });
  __syncthreads();  // (the buffer and flags of this segment are used again)
  });
}

// ---- wide tiles (bf16, more than 64 query rows that share their keys): four waves of 32 rows each, all on the same keys, so that
// a tile of 64 keys is read from memory once for 128 rows, straight into LDS and two tiles ahead.  S(j+1) = K(j+1) Q^T runs beside
// the exponentials of S(j), O += V(j)^T P(j) beside the first half of those of S(j+1): an instruction stream that gives the matrix
// cores and the vector unit independent work.  The softmax reference is the maximum of the first tile a row sees and is raised only
// where a row sum says that it has to be (a probability of 2^40): numerator and denominator carry the same factor, so nothing is
// lost by a reference that is too low.
// Bound by the matrix cores, busy 52 to 56 % of the time (tiles whose last waves have no rows, starts and ends of pieces).  32 sessions
// with trees of 24 to 64 tokens over 2048 to 16384 keys (G 4: 1.31 GB, 243 GF): 475 us, 512 TF, or 770 with the products of the
// probabilities' second halves; 64 tokens over 32768 keys (G 8) 112 us.  A small call is made of trips to memory: 26 tokens over 3001
// keys 18.1 us, 2.2 to find the piece, 2.5 for ids and first tiles, 1.6 a tile, 1.9 at the end, 4.6 for the join.
constexpr int kWideKeys = 64;
constexpr float kRaiseSum = 1.0995116e12f;  // 2^40

// A wide tile's piece in the workspace: the registers of its 256 threads, then (m, l) of each, then which piece of what it is (the
// join reads that instead of working it out again: 1.5 us)
struct WideNote {
  int32_t cu, P, N, tile, index, count, stride, reserved;  // count 0: no piece
};
template <int D>
constexpr int kWideSlot = 128 * D + 512 + (int)(sizeof(WideNote) / 4);
template <int D>
__device__ __forceinline__ float* wide_slot(const TreeParams& p, int64_t piece, int kvh) {
  return p.parts + (piece * p.n_kv_heads + kvh) * (int64_t)kWideSlot<D>;
}

template <int D>
__global__ __launch_bounds__(256, 2) void tree_wide_kernel(const TreeParams p) {
  typedef __bf16 T;
  typedef TileLds<D> Lds;
  constexpr int BM = 128, KB = kWideKeys, NS = D / 16, NT = D / 32;
  constexpr int kFrags = 4 * NT;  // operands of V a tile: (32-key half, 16-key step, 32-column tile)
  constexpr int kAhead = 4;       // operands read from LDS ahead of their use
  // (arrays of their own, so that the compiler can tell which loads an LDS read has to wait for)
  __shared__ __attribute__((aligned(16))) char K0[Lds::kBytes];
  __shared__ __attribute__((aligned(16))) char K1[Lds::kBytes];
  __shared__ __attribute__((aligned(16))) char V0[Lds::kBytes];
  __shared__ __attribute__((aligned(16))) char V1[Lds::kBytes];
  __shared__ float again_lds[4][2 * D];

  const int Hkv = p.n_kv_heads;
  const int G = p.group;
  int kvh, piece;
  split_block(p, blockIdx.x, kvh, piece);
  TreePiece it;
  const bool found = find_piece<BM, KB>(p, G, piece, it);
  if (p.cut && threadIdx.x == 0)
    *reinterpret_cast<WideNote*>(wide_slot<D>(p, piece, kvh) + 128 * D + 512) =
        found ? WideNote{it.cu, it.P, it.N, it.tile, it.index, it.count, it.stride, 0} : WideNote{};
  if (!found) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31;  // query row of this lane within its wave's; also its row of the K operand
  const int kg = lane >> 5;
  const int cu = it.cu, P = it.P, N = it.N;
  const unsigned row0 = (unsigned)it.tile * BM;
  const int n_rows = (int)min((unsigned)BM, (unsigned)N * (unsigned)G - row0);
  const bool works = wave * 32 < n_rows;  // (a wave without rows only moves its share of the tiles)
  const int prefix_tiles = P / KB + (P % KB != 0), full_tiles = P / KB;
  const int begin = it.block0;
  int end = it.block1;

  const unsigned my_row = row0 + min(wave * 32 + n, n_rows - 1);
  const int tok = token_of(p, my_row);
  const uint32_t* const mask_row = p.mask + (int64_t)(cu + tok) * p.mask_words;
  bf16x8 q[NS];
  {
    const T* const qp = (const T*)p.q + ((int64_t)(cu + tok) * p.n_q_heads + kvh * G + (int)(my_row - (unsigned)tok * G)) * D;
#pragma unroll
    for (int st = 0; st < NS; ++st) q[st] = *reinterpret_cast<const bf16x8*>(qp + 16 * st + 8 * kg);
  }

  // ---- memory -> LDS.  Block ids of the wave's loads: asked for by lanes an iteration before they are needed, then made addresses
  // and moved to scalar registers (asking for the value at once would also wait for the tiles under way).
  const bool has_table = p.table != nullptr && p.table_stride > 0;
  const int32_t* const table_row = p.table + (int64_t)it.s * p.table_stride;
  const unsigned row_bytes = (unsigned)(Hkv * D * (int)sizeof(T));
  const char* const k_pool = reinterpret_cast<const char*>((const T*)p.k_layer + kvh * D);
  const char* const v_pool = reinterpret_cast<const char*>((const T*)p.v_layer + kvh * D);
  const char* const k_fresh = reinterpret_cast<const char*>((const T*)p.k_new + (int64_t)cu * Hkv * D + kvh * D);
  const char* const v_fresh = reinterpret_cast<const char*>((const T*)p.v_new + (int64_t)cu * Hkv * D + kvh * D);
  constexpr int kLoads = Lds::kLoads;
  auto my_key = [&](int tile) {  // of lane i: the first of load i % kLoads, of tile or the one behind it
    return (unsigned)(tile + lane / kLoads % 2) * KB + (unsigned)Lds::row_of(lane % kLoads, wave, 0);
  };
  auto ask_ids = [&](int tile) {
    const unsigned at = table_place(p, my_key(tile));
    return has_table ? table_row[(int)min(at, (unsigned)p.table_stride - 1)] : -1;
  };
  auto find_rows = [&](int tile, int ids) {
    const unsigned key = my_key(tile);
    return rows_at(p, key, table_place(p, key), ids, row_bytes);
  };
  int64_t rows_k[kLoads], rows_v[kLoads];  // of this wave's loads
  int asked;
  const unsigned lane_off = (unsigned)(lane / (D / 8)) * row_bytes + (unsigned)Lds::chunk_of(Lds::row_of(0, wave, lane), lane) * 16u;
  auto issue_tile = [&](const char* pool, const char* fresh, char* buf, int tile, const int64_t (&rows)[kLoads]) {
    if (__builtin_expect(tile < full_tiles, 1)) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const bool known = rows[i] >= 0;  // (else rows of zeros)
        load_lds16<0>(known ? pool + rows[i] : reinterpret_cast<const char*>(kNoRow),
                      known ? lane_off : (unsigned)(lane % (D / 8)) * 16u, buf + Lds::at(i, wave));
      }
    } else {
      // the prefix's last tile, or one of the tree: in place of rows that do not exist the last one that does (no row sees them)
      int l = lane;
      asm volatile("" : "+v"(l));  // (its pieces of addresses are worked out here: no registers for them in the loop)
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int row = Lds::row_of(i, wave, l), first_row = Lds::row_of(i, wave, 0);
        const unsigned in_row = (unsigned)Lds::chunk_of(row, l) * 16u;
        const char* base = reinterpret_cast<const char*>(kNoRow);
        unsigned off = in_row;
        if (tile < prefix_tiles) {
          const int first = tile * KB + first_row;
          if (first < P && rows[i] >= 0) {
            base = pool + rows[i];
            off += (unsigned)min(row - first_row, P - 1 - first) * row_bytes;
          }
        } else {
          const int first = (tile - prefix_tiles) * KB;
          base = fresh + (uint64_t)first * row_bytes;
          off += (unsigned)min(row, N - 1 - first) * row_bytes;
        }
        load_lds16<0>(base, off, buf + Lds::at(i, wave));
      }
    }
  };

  // ---- LDS reads.  K: lane (n, kg) reads chunk 2 * st + kg of key row key_of_row(n) (+ 32 for the second half).  V: 16 lanes read
  // 4 rows x 32 bytes and each gets one column, i.e. 4 consecutive keys of it.
  const int krow = key_of_row(n);
  int k_off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_off[i] = Lds::place(krow, D == 128 ? 4 * i + kg : 2 * i + kg);
  auto k_frag = [&](const char* buf, int st, int kb) { return Lds::k_frag(buf, k_off, st, kb); };
  const int i16 = lane & 15;
  int v_off[4];  // 128: by column tile; 64: by column tile and half of the 8 keys
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int dt = D == 128 ? i : i >> 1, half = D == 128 ? 0 : i & 1;
    const int row = 8 * kg + 4 * half + (i16 >> 2);
    v_off[i] = Lds::place(row, 4 * dt + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) + 8 * (i16 & 1);
  }
  auto v_frag = [&](const char* buf, int g) { return Lds::v_frag(buf, v_off, g); };

  f32x16 o[NT];
#pragma unroll
  for (int dt = 0; dt < NT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.f;
  float m_ref = -INFINITY, l_run = 0.f;  // the reference in log2 units, this lane's share of the sum
  const float cs = p.scale * 1.4426950408889634f;

  auto scores = [&](const char* buf, f32x16 (&sc)[2]) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[kb][e] = 0.f;
#pragma unroll
    for (int st = 0; st < NS; ++st)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(buf, st, kb), q[st], sc[kb], 0, 0, 0);
  };
  // Keys that the lane's row does not see, given the mask's words of the tile
  auto ask_words = [&](int tile, uint32_t (&words)[2]) {
    if (tile < full_tiles) return;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) words[kb] = mask_word(p, mask_row, tile < prefix_tiles ? -1 : 2 * (tile - prefix_tiles) + kb);
  };
  auto hide = [&](f32x16 (&sc)[2], int tile, const uint32_t (&words)[2]) {
    if (tile < full_tiles) return;
    const int left = tile < prefix_tiles ? P - tile * KB : N - (tile - prefix_tiles) * KB;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      const uint32_t bits = seen_keys(left - 32 * kb, words[kb]) >> (8 * kg);
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[kb][e] = score_if(bits, 16 * (e >> 3) + (e & 7), sc[kb][e]);
    }
  };
  // The reference := max(reference, maximum of this tile); returns the factor for what has been accumulated
  auto raise_reference = [&](const f32x16 (&sc)[2], float& ref) {
    float mx = sc[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[kb][e]);
    const float m_new = fmaxf(m_ref, max_across_halves(mx) * cs);
    const float a = m_ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_ref - m_new);
    m_ref = m_new;
    ref = m_new == -INFINITY ? 0.f : m_new;
    return a;
  };
  f32x16 s_even[2], s_odd[2];  // scores of the even and of the odd tiles, counted from the first
  bf16x8 hi[2][2], lo[2][2];   // P(j)
  float ref = 0.f, sum_first = 0.f;
  asked = ask_ids(begin);
  if (N > KB)  // (at least one tile: its rows are told that they saw nothing)
    end = min(end, max(prefix_tiles + tree_blocks_seen<KB>(p, cu, N, row0, n_rows), begin + 1));
  {
    const int64_t found = find_rows(begin, asked);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      rows_k[i] = lane_value(found, i);
      rows_v[i] = lane_value(found, kLoads + i);  // (of the second tile)
    }
  }
  uint32_t words_first[2] = {};
  ask_words(begin, words_first);
  issue_tile(k_pool, k_fresh, K0, begin, rows_k);
  issue_tile(v_pool, v_fresh, V0, begin, rows_k);
  if (begin + 1 < end) issue_tile(k_pool, k_fresh, K1, begin + 1, rows_v);
  // The first product needs K0 only: V0 and K1, issued after it, may still be on their way (loads return in order)
  if (begin + 1 < end)
    __builtin_amdgcn_s_waitcnt(0x0F70 | (2 * Lds::kLoads));
  else
    __builtin_amdgcn_s_waitcnt(0x0F70 | Lds::kLoads);
  __syncthreads();
  if (works) {
    scores(K0, s_even);
    hide(s_even, begin, words_first);
    raise_reference(s_even, ref);
    sum_first = probabilities(s_even[0], cs, ref, hi[0], lo[0]);
  }
  asked = ask_ids(begin + 2);
  auto arrived = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's loads into LDS have landed
    __syncthreads();
  };
  arrived();

  // P(j)'s second half and the end of its statistics; a row without a reference yet, or with one that is far too low, gets one
  auto rest_of_tile = [&](const f32x16 (&sc)[2]) {
    float sum = sum_first + probabilities(sc[1], cs, ref, hi[1], lo[1]);
    return sum;
  };
  auto settle = [&](const f32x16 (&sc)[2], float sum) {
    if (__any(!(sum <= kRaiseSum) || m_ref == -INFINITY)) {
      const float a = raise_reference(sc, ref);
      l_run *= a;
#pragma unroll
      for (int dt = 0; dt < NT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= a;
      sum = probabilities(sc[0], cs, ref, hi[0], lo[0]) + probabilities(sc[1], cs, ref, hi[1], lo[1]);
    }
    l_run += sum;
  };

  auto iteration = [&](const int j, auto parity) {
    constexpr int PAR = decltype(parity)::value;
    char* const k_same = PAR ? K1 : K0;   // held K(j), free now: receives K(j+2)
    char* const k_other = PAR ? K0 : K1;  // holds K(j+1)
    char* const v_same = PAR ? V1 : V0;   // holds V(j)
    char* const v_other = PAR ? V0 : V1;  // held V(j-1), free now: receives V(j+1)
    f32x16(&s_cur)[2] = PAR ? s_odd : s_even;  // S(j)
    f32x16(&s_nxt)[2] = PAR ? s_even : s_odd;  // receives S(j+1)
    {
      const int64_t found = find_rows(j + 2, asked);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) rows_k[i] = lane_value(found, i);
    }
    asked = ask_ids(j + 3);
    uint32_t words[2] = {};
    ask_words(j + 1, words);
    issue_tile(v_pool, v_fresh, v_other, j + 1, rows_v);
    if (j + 2 < end) issue_tile(k_pool, k_fresh, k_same, j + 2, rows_k);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) rows_v[i] = rows_k[i];
    if (works) {
      // In explicit slots, between which nothing moves (the compiler's own order reads an operand right before its use and puts
      // the exponentials behind the products): the LDS read of the operand four slots ahead, one matrix instruction of S(j+1),
      // its share of the 16 exponentials of P(j)'s second half.
      float sums_a[2] = {0.f, 0.f};
      {
        constexpr int kPer = 16 / (2 * NS);
        bf16x8 frag[2 * NS];
        float pe[16];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e) s_nxt[kb][e] = 0.f;
#pragma unroll
        for (int g = 0; g < kAhead; ++g) frag[g] = k_frag(k_other, g >> 1, g & 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < 2 * NS; ++g) {
          if (g + kAhead < 2 * NS) frag[g + kAhead] = k_frag(k_other, (g + kAhead) >> 1, (g + kAhead) & 1);
          s_nxt[g & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[g], q[g >> 1], s_nxt[g & 1], 0, 0, 0);
#pragma unroll
          for (int k = kPer * g; k < kPer * (g + 1); ++k) {
            pe[k] = __builtin_amdgcn_exp2f(fmaf(s_cur[1][k], cs, -ref));
            asm volatile("" : "+v"(pe[k]));  // (in this slot, not next to its use)
            sums_a[k & 1] += pe[k];
            if (k & 1) {
              put_pair(hi[1][k >> 3], (k & 7) - 1, pe[k - 1], pe[k]);
              put_pair(lo[1][k >> 3], (k & 7) - 1, pe[k - 1] - upper_part(pe[k - 1]), pe[k] - upper_part(pe[k]));
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) asm volatile("" : "+v"(hi[1][u]), "+v"(lo[1][u]));  // (computed here, not past the branch)
      }
      float sum = sum_first + sums_a[0] + sums_a[1];
      asm volatile("" : "+v"(sum));
      settle(s_cur, sum);
      hide(s_nxt, j + 1, words);
      // O += V(j)^T P(j) beside the first half of P(j+1): in every slot the LDS reads of the operand some slots ahead, the two
      // products of one operand and their share of the 16 exponentials
      bf16x8 hi_first[2], lo_first[2];
      bf16x8 frag[kFrags];
      constexpr int kPer = 16 / kFrags;  // exponentials of a slot
      float pe[16], sums[2] = {0.f, 0.f};
#pragma unroll
      for (int g = 0; g < kAhead; ++g) frag[g] = v_frag(v_same, g);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int g = 0; g < kFrags; ++g) {
        if (g + kAhead < kFrags) frag[g + kAhead] = v_frag(v_same, g + kAhead);
        const int step = g / NT;
        o[g % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[g], hi[step >> 1][step & 1], o[g % NT], 0, 0, 0);
#pragma unroll
        for (int k = kPer * g; k < kPer * (g + 1); ++k) {
          pe[k] = __builtin_amdgcn_exp2f(fmaf(s_nxt[0][k], cs, -ref));
          asm volatile("" : "+v"(pe[k]));  // (in this slot, not next to its use)
          sums[k & 1] += pe[k];
        }
        o[g % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[g], lo[step >> 1][step & 1], o[g % NT], 0, 0, 0);
#pragma unroll
        for (int k = kPer * g; k < kPer * (g + 1); ++k)
          if (k & 1) {
            put_pair(hi_first[k >> 3], (k & 7) - 1, pe[k - 1], pe[k]);
            put_pair(lo_first[k >> 3], (k & 7) - 1, pe[k - 1] - upper_part(pe[k - 1]), pe[k] - upper_part(pe[k]));
          }
        __builtin_amdgcn_sched_barrier(0);
      }
      sum_first = sums[0] + sums[1];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        hi[0][u] = hi_first[u];
        lo[0][u] = lo_first[u];
        asm volatile("" : "+v"(hi[0][u]), "+v"(lo[0][u]));
      }
    }
    arrived();
  };
  for (int j = begin; j + 1 < end; j += 2) {
    iteration(j, std::integral_constant<int, 0>{});
    if (j + 2 < end) iteration(j + 1, std::integral_constant<int, 1>{});
  }
  // The last tile has no successor
  if (works) {
    const bool odd = (end - 1 - begin) & 1;
    if (odd) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) s_even[kb] = s_odd[kb];
    }
    const char* const v_last = odd ? V1 : V0;
    settle(s_even, rest_of_tile(s_even));
#pragma unroll
    for (int g = 0; g < kFrags; ++g) {
      const int step = g / NT;
      const bf16x8 v = v_frag(v_last, g);
      o[g % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, hi[step >> 1][step & 1], o[g % NT], 0, 0, 0);
      o[g % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, lo[step >> 1][step & 1], o[g % NT], 0, 0, 0);
    }
  }
  // ---- results, from the registers they are in: a lane has columns 32 dt + 8 i + 4 kg .. + 3 of its row at o[dt][4 i ..].  A row
  // with a value that is not finite, or with scores beyond what the loop's arithmetic is made for, is worked out again by itself
  // (see finish_tile), from its q, which `out` may be: it is not written here.
  const float l = sum_across_halves(l_run);
  const bool whole = it.count == 1;
  float* const slot = whole ? nullptr : wide_slot<D>(p, piece, kvh);
  unsigned again = 0;
  if (works) {
    float not_finite = 0.f;  // 0 times every value: 0, or NaN
#pragma unroll
    for (int dt = 0; dt < NT; ++dt)
#pragma unroll
      for (int e = 0; e < 16; ++e) not_finite = fmaf(o[dt][e], 0.f, not_finite);
    not_finite = sum_across_halves(not_finite);
    const bool bad = (not_finite != 0.f && l == l && l != 0.f) || (fabsf(m_ref) > kLargestScore && m_ref != -INFINITY);
    const bool exists = wave * 32 + n < n_rows;
    again = (unsigned)__ballot(bad && exists);
    float scale = 1.0f, none = 0.f;
    if (whole) {
      scale = l == 0.f ? 0.f : 1.0f / l;
      if (l == 0.f) none = nothing_seen(p, it, tok);
    }
    // (a row without any probability: whatever values the product brought in are not its own)
    if (whole) {
      if (exists && !bad) {
        typedef T vec __attribute__((ext_vector_type(4)));
        T* const op =
            (T*)p.out + ((int64_t)(cu + tok) * p.n_q_heads + kvh * G + (int)(my_row - (unsigned)tok * G)) * D + 4 * kg;
#pragma unroll
        for (int dt = 0; dt < NT; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            vec y;
#pragma unroll
            for (int v = 0; v < 4; ++v) y[v] = (T)(l == 0.f ? none : o[dt][4 * i + v] * scale);
            *reinterpret_cast<vec*>(op + 32 * dt + 8 * i) = y;
          }
      }
    } else {
      // as the registers are, 16 bytes per lane: whole lines, nothing to arrange
#pragma unroll
      for (int dt = 0; dt < NT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x4 x{o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
          if (l == 0.f) x = f32x4{0.f, 0.f, 0.f, 0.f};
          *reinterpret_cast<f32x4*>(slot + ((dt * 4 + i) * 256 + tid) * 4) = x;
        }
      *reinterpret_cast<f32x2*>(slot + BM * D + 2 * tid) = f32x2{m_ref, l};
    }
  }
  // (no barrier: other waves' stores are not waited for, their rows and the tile buffers not touched)
  float* const own = again_lds[wave];
  for (unsigned left = __builtin_amdgcn_readfirstlane(again); left; left &= left - 1) {
    const int r = __builtin_ctz(left);
    const unsigned row = row0 + wave * 32 + r, tk = (unsigned)token_of(p, row);
    const int h = kvh * G + (int)(row - tk * G);
    float m, lr;
    row_by_lanes<T, D, KB, 64>(p, it, (int)tk, h, own, m, lr);
    if (whole) {
      T* const op = (T*)p.out + ((int64_t)(cu + (int)tk) * p.n_q_heads + h) * D;
      const float none = lr == 0.f ? nothing_seen(p, it, (int)tk) : 0.f;
      for (int c = lane; c < D; c += 64) op[c] = (T)(lr == 0.f ? none : own[D + c] * (1.0f / lr));
    } else {
      for (int c = lane; c < D; c += 64)
        slot[(c / 8 * 256 + wave * 64 + 32 * (c / 4 & 1) + r) * 4 + (c & 3)] = own[D + c];
      if (lane < 2) *reinterpret_cast<f32x2*>(slot + BM * D + 2 * (wave * 64 + 32 * lane + r)) = f32x2{m, lr};
    }
  }
}

// ---- joins the pieces of cut tiles: out = sum_c f_c O_c / sum_c f_c l_c, f_c = e^(m_c - max_c m_c).
// The O_c are finite each, but as large as the type takes where the values are, so that the sum of a few would overflow: they are
// added up 2^12 times smaller, which is more than a tile has pieces (1025 at most).  A power of two changes no bit of the quotient,
// but where f_c is below 2^-114: there the product with it has fewer bits than a float, as f_c itself has from 2^-126 on.
constexpr float kJoinShrink = 0x1p-12f, kJoinGrow = 0x1p12f;

// AT_ONCE pieces, of which the first `left` count, into a running maximum, sum and row (kJoinShrink of it)
template <typename T, int AT_ONCE>
__device__ __forceinline__ void add_pieces(float& M, float& L, f32x4& o, const f32x4 (&oc)[AT_ONCE], const f32x2 (&ml)[AT_ONCE],
                                           int left) {
  float m_new = M;
#pragma unroll
  for (int k = 0; k < AT_ONCE; ++k) m_new = fmaxf(m_new, ml[k][0]);
  const float a = M == -INFINITY ? 0.f : exp_of<T>(M - m_new);
  M = m_new;
  L = L == L ? L * a : L;
  o *= a;
#pragma unroll
  for (int k = 0; k < AT_ONCE; ++k) {
    const float m = ml[k][0], l = ml[k][1];
    // (a piece without a maximum has no key that the row sees, or scores that are NaN: then so is its sum)
    const float f = k >= left ? 0.f : m == -INFINITY ? (l == l ? 0.f : 1.f) : exp_of<T>(m - M);
    if (f != 0.f) {
      L += l * f;
      o += oc[k] * (kJoinShrink * f);
    }
  }
}

// Each of a tile's pieces has a workgroup here too, which joins an equal share of the tile's rows.  A join is nothing but trips to
// memory: D / 4 lanes take a row's columns of eight pieces at a time, and where there are fewer rows than such groups of lanes,
// several share a row.
template <typename T, int D, int BM, typename Slot>
__device__ __forceinline__ void join_rows(const TreeParams& p, const PartNote& it, int kvh, Slot slot_of) {
  constexpr int kLanes = D / 4, kSubs = 256 / kLanes, kAtOnce = 8;
  __shared__ f32x4 part_o[kSubs][kLanes];
  __shared__ float part_m[kSubs], part_l[kSubs];
  const int tid = threadIdx.x, sub = tid / kLanes, c0 = 4 * (tid % kLanes);
  const int G = p.group;
  const unsigned row0 = (unsigned)it.tile * BM;
  const int n_rows = (int)min((unsigned)BM, (unsigned)it.N * (unsigned)G - row0);
  const int r0 = (int)((int64_t)n_rows * it.index / it.count), r1 = (int)((int64_t)n_rows * (it.index + 1) / it.count);
  int at_once = 1;  // rows
  while (at_once < kSubs && at_once < r1 - r0) at_once *= 2;
  const int share = sub / at_once, shares = kSubs / at_once;
  for (int rb = r0; rb < r1; rb += at_once) {
    const int r = rb + sub % at_once;
    float M = -INFINITY, L = 0.f;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    if (r < r1) {
      for (int c = share; c < it.count; c += kAtOnce * shares) {
        f32x4 oc[kAtOnce];
        f32x2 ml[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {  // (past the last piece: it again, without weight)
          const float* const slot = slot_of(min(c + k * shares, it.count - 1));
          oc[k] = *reinterpret_cast<const f32x4*>(slot + r * D + c0);
          ml[k] = f32x2{slot[BM * D + r], slot[BM * D + BM + r]};
        }
        add_pieces<T, kAtOnce>(M, L, o, oc, ml, (it.count - c + shares - 1) / shares);
      }
    }
    if (shares > 1) {
      if (r < r1) {
        part_o[sub][tid % kLanes] = o;
        part_m[sub] = M;
        part_l[sub] = L;
      }
      __syncthreads();
      if (share == 0 && r < r1) {
        float top = M;
        for (int k = 1; k < shares; ++k) top = fmaxf(top, part_m[sub + k * at_once]);
        float f = M == -INFINITY ? (L == L ? 0.f : 1.f) : exp_of<T>(M - top);
        L *= f;
        o *= f;
        for (int k = 1; k < shares; ++k) {
          const float mk = part_m[sub + k * at_once], lk = part_l[sub + k * at_once];
          f = mk == -INFINITY ? (lk == lk ? 0.f : 1.f) : exp_of<T>(mk - top);
          L += lk * f;
          o += part_o[sub + k * at_once][tid % kLanes] * f;
        }
      }
      __syncthreads();
    }
    if (share == 0 && r < r1) {
      const unsigned row = row0 + r, tok = (unsigned)token_of(p, row);
      const float none = L == 0.f ? nothing_seen(p, it, (int)tok) : 0.f;
      typedef T vec __attribute__((ext_vector_type(4)));
      vec y;
#pragma unroll
      for (int v = 0; v < 4; ++v) y[v] = (T)(L == 0.f ? none : o[v] * (kJoinGrow / L));
      T* const op = (T*)p.out + ((int64_t)(it.cu + (int)tok) * p.n_q_heads + kvh * G + (int)(row - tok * G)) * D;
      *reinterpret_cast<vec*>(op + c0) = y;
    }
  }
}

// Wide tiles: the workgroups of the tile's pieces take their shares of the 16-byte vectors of a thread, thread by thread as they were
// written.  32 wide trees (1640 pieces of 64 KB) take 23 to 25 us, one user's 24 pieces 4.6.
template <int D>
__global__ __launch_bounds__(256) void tree_join_wide_kernel(const TreeParams p) {
  typedef __bf16 T;
  typedef T vec __attribute__((ext_vector_type(4)));
  constexpr int BM = 128, kVecs = D / 8, kAtOnce = 8;
  const int Hkv = p.n_kv_heads, G = p.group;
  int kvh, piece;
  split_block(p, blockIdx.x, kvh, piece);
  const WideNote it = *reinterpret_cast<const WideNote*>(wide_slot<D>(p, piece, kvh) + 128 * D + 512);
  const int mine = it.index + it.count * (int)blockIdx.y;
  if (it.count <= 1 || mine >= kVecs) return;
  const int tid = threadIdx.x, r = (tid >> 6) * 32 + (tid & 31);
  const unsigned row0 = (unsigned)it.tile * BM;
  const int n_rows = (int)min((unsigned)BM, (unsigned)it.N * (unsigned)G - row0);
  if (r >= n_rows) return;
  const float* const first = wide_slot<D>(p, piece - (int64_t)it.index * it.stride, kvh);
  const int64_t stride = (int64_t)it.stride * Hkv * kWideSlot<D>;
  const unsigned row = row0 + r, tok = (unsigned)token_of(p, row);
  T* const op = (T*)p.out + ((int64_t)(it.cu + (int)tok) * p.n_q_heads + kvh * G + (int)(row - tok * G)) * D + 4 * (tid >> 5 & 1);
  for (int v = mine; v < kVecs; v += it.count * (int)gridDim.y) {
    float M = -INFINITY, L = 0.f;
    f32x4 o{0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < it.count; c += kAtOnce) {
      f32x4 oc[kAtOnce];
      f32x2 ml[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {  // (past the last piece: it again, without weight)
        const float* const slot = first + min(c + k, it.count - 1) * stride;
        oc[k] = *reinterpret_cast<const f32x4*>(slot + (v * 256 + tid) * 4);
        ml[k] = *reinterpret_cast<const f32x2*>(slot + BM * D + 2 * tid);
      }
      add_pieces<T, kAtOnce>(M, L, o, oc, ml, it.count - c);
    }
    const float none = L == 0.f ? nothing_seen(p, it, (int)tok) : 0.f;
    vec y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (T)(L == 0.f ? none : o[e] * (kJoinGrow / L));
    *reinterpret_cast<vec*>(op + 8 * v) = y;
  }
}

// The same for ranges: a workgroup for each of the two places of a range
template <typename T, int D, int BM>
__global__ __launch_bounds__(256) void tree_join_ranges_kernel(const TreeParams p) {
  int kvh, place;
  split_block(p, blockIdx.x, kvh, place);
  const PartNote it = *part_note<BM, D>(p, place, kvh);
  if (it.count <= 1) return;
  // (the second and later parts of a tile start with their ranges, in the first of their two places)
  const float* const own = part_slot<BM, D>(p, it.own, kvh);
  const float* const later = part_slot<BM, D>(p, it.own & ~1, kvh);
  const int64_t stride = it.step * (int64_t)p.n_kv_heads * kPartSlot<BM, D>;
  join_rows<T, D, BM>(p, it, kvh, [&](int c) { return c == 0 ? own : later + c * stride; });
}

// ------------------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------------------
constexpr int kWideSlots = 512;    // workgroups of wide tiles that are on the chip at once: two per compute unit
// and that the key axis is cut for at most, all kv-heads together: two rounds level out what sessions differ by (32 wide trees take
// 1.5 % longer with one)
constexpr int kWidePieces = 1024;
constexpr int kRanges = 256;       // the same for ranges: one workgroup per compute unit (twice as many of half the waves: equal)
constexpr int kStreamWaves = 8;
// Parts of a wide tile's join, as far as it does not have as many pieces (8: 1 % slower over calls of many rows, none 1.4)
constexpr int kJoinParts = 16;

struct TreePlan {
  bool wide;           // 128-row tiles through LDS
  int waves;           // streams: of a workgroup
  unsigned join_parts; // workgroups that join what one has produced
  int rw;              // else: waves side by side on the rows
  int64_t pieces;      // per kv-head
  bool aligned;        // narrow tiles in pieces
  int32_t c_min;       // key blocks
  bool cut;
  int64_t bytes;
};

// The rows of a load lie in one block of the cache and a block fits 32 bits: rows can be addressed by groups
static bool grouped_rows(const symph_kv_cache* c) {
  if (c->block_stride * (int64_t)elem_bytes_of(c->dtype) > 0x7FFFFFFFLL) return false;
  return c->block_size % (c->dtype == SYMPH_BF16 && c->head_dim == 128 ? TileLds<128>::kGroupRows : 8) == 0;
}

// Everything that follows from host-side values alone; the workspace query and the call agree on it.
static bool plan_tree(TreePlan& pl, const symph_kv_cache* c, int32_t n_sessions, int32_t n_q_heads, int32_t total,
                      int32_t max_new, int32_t max_prefix) {
  const int R = c->dtype == SYMPH_BF16 ? 32 : 16;
  const int64_t G = n_q_heads / c->n_kv_heads;
  const int64_t rows = (int64_t)max_new * G;
  pl.aligned = false;
  pl.wide = c->dtype == SYMPH_BF16 && rows > 64 && grouped_rows(c);
  pl.rw = rows <= R ? 1 : rows <= 2 * R ? 2 : 4;
  const int64_t BM = pl.wide ? 128 : (int64_t)R * pl.rw, KB = pl.wide || (R == 32 && c->head_dim == 64) ? 64 : R;
  const int64_t tiles = (int64_t)total * G / BM + n_sessions;  // at least as many as there are
  // (more rows or tiles than a grid takes: what follows stays within 64 bits)
  if (rows > 0x7FFFFFFFLL || (int64_t)total * G > 0x7FFFFFFFLL || tiles > 0x7FFFFFFFLL / c->n_kv_heads) return false;
  const int64_t blocks = ceil_div64(max_prefix, KB) + ceil_div64(max_new, KB);
  // A second launch that joins pieces takes 4 to 5 us, as long as a workgroup does for `uncut` blocks; where it is worth that, pieces
  // are as short as pays: a wide tile's 64 keys are 1.4 us of its 6, a workgroup of streams is full with a block per wave.
  const int64_t uncut = pl.wide ? 5 : R == 16 ? (c->head_dim == 64 ? 20 : 12) : c->head_dim == 64 ? 12 : 20;
  pl.c_min = pl.wide ? 2 : 4;
  // Else eight waves fill a compute unit, fewer let it take more workgroups, for tiles that keep few waves busy or are many.  A round
  // of workgroups takes some 6 us and 2.5 for every block of a wave, and a cut batch of many sessions some 40 us beside its bytes
  // (parts of several tiles per workgroup, their results, the join).  So it stays whole where the rounds take less than that, or the
  // tiles are so many that a long one at the end is a small part (249 sessions of up to 887 keys 160 -> 119 us, 191 fp32 trees of
  // 247 tokens 1430 -> 1200).
  pl.waves = kStreamWaves;
  bool brief = false;
  if (!pl.wide && (R == 16 || grouped_rows(c))) {
    const int64_t all = (pl.rw <= 2 ? n_sessions : tiles) * c->n_kv_heads;  // (few rows: a session is one tile)
    int64_t best = INT64_MAX;
    for (int w = kStreamWaves; w >= std::max(2, pl.rw); w /= 2) {
      const int64_t takes = ceil_div64(all, kRanges * kStreamWaves / w) * (12 + 5 * ceil_div64(blocks, w / pl.rw));
      if (takes < best) best = takes, pl.waves = w;
    }
    brief = (all >= kRanges / 2 && best <= 80) || (all >= 2 * kRanges && blocks * kRanges <= R / 2 * all);
    if (blocks > uncut && !brief) pl.waves = kStreamWaves;
  }
  // Wide tiles that fill the chip as they are, and are not long: a tail costs less than pieces do (their search, results and join;
  // 144 sessions of 38 tokens and up to 400 keys 93 us against 117).
  const bool many = pl.wide && (int64_t)total * G / BM * c->n_kv_heads >= kWideSlots / 2 && blocks <= 48;
  const int64_t per_tile = blocks <= uncut || brief || many ? 1 : ceil_div64(blocks, pl.c_min);
  const int64_t target = ceil_div64(pl.wide ? kWidePieces : kRanges, c->n_kv_heads);
  if (pl.wide) {
    const int64_t more = per_tile <= 1 ? 0 : tiles >= target ? target : std::min(tiles * (per_tile - 1), target);
    pl.cut = more > 0;
    pl.pieces = tiles + more;
    pl.join_parts = (unsigned)std::clamp<int64_t>(kJoinParts * tiles / pl.pieces, 1, 4);
  } else {
    pl.cut = per_tile > 1;
    pl.pieces = pl.cut ? std::min(tiles * per_tile, target) : tiles;
    // A range that runs into another session costs some 8 us more, a piece that ends with its tile leaves workgroups unlike: half a
    // piece of a tile's share of 5 us for every block of a wave.  (Nine sessions of up to 940 keys 20.3 -> 14.6 us, eight of up to
    // 4000 37 -> 33; 113 of up to 20 000 would take 210 against 170.  One session's ranges are its pieces.)
    // Ranges cover whatever there is; of pieces every tile takes one at least, so there have to be as many as tiles of any lengths,
    // not of those that max_new says.  (Where a session is one tile that is so: then tiles <= 2 * count.)
    const int64_t count = pl.rw <= 2 ? n_sessions : tiles;
    pl.aligned = pl.cut && R == 32 && n_sessions > 1 && tiles <= pl.pieces && 2 * count <= pl.pieces &&
                 count * count * blocks <= 2 * kStreamWaves * pl.pieces * pl.pieces;
  }
  pl.bytes = !pl.cut ? 0 : pl.wide ? pl.pieces * c->n_kv_heads * (c->head_dim == 128 ? kWideSlot<128> : kWideSlot<64>) * 4
                                   : 2 * pl.pieces * c->n_kv_heads * (BM * (c->head_dim + 2) * 4 + (int64_t)sizeof(PartNote));
  if (ceil_div64(rows, BM) * blocks > kMostWork) return false;
  return grid_takes(pl.pieces * c->n_kv_heads, pl.wide ? 256 : 64 * pl.waves) &&
         (!pl.cut || pl.wide || grid_takes(2 * pl.pieces * c->n_kv_heads, 256));  // (the join of ranges)
}

template <typename T, int D, int RW>
static void launch_tree(const TreeParams& p, int64_t pieces, int waves, hipStream_t stream) {
  const dim3 grid((unsigned)(pieces * p.n_kv_heads)), join((unsigned)(2 * pieces * p.n_kv_heads));
  if constexpr (sizeof(T) == 2) {
    if (p.group_bytes == 0)
      hipLaunchKernelGGL((tree_stream_kernel<D, RW, kStreamWaves, false>), grid, dim3(64 * kStreamWaves), 0, stream, p);
    else if constexpr (RW <= 2) {  // (more rows: wide tiles)
      if (waves == 2)
        hipLaunchKernelGGL((tree_stream_kernel<D, RW, 2, true>), grid, dim3(128), 0, stream, p);
      else if (waves == 4)
        hipLaunchKernelGGL((tree_stream_kernel<D, RW, 4, true>), grid, dim3(256), 0, stream, p);
      else
        hipLaunchKernelGGL((tree_stream_kernel<D, RW, kStreamWaves, true>), grid, dim3(64 * kStreamWaves), 0, stream, p);
    }
    if (p.cut) hipLaunchKernelGGL((tree_join_ranges_kernel<T, D, 32 * RW>), join, dim3(256), 0, stream, p);
  } else {
    if constexpr (RW <= 2) {
      if (waves == 2) hipLaunchKernelGGL((tree_fp32_kernel<D, RW, 2>), grid, dim3(128), 0, stream, p);
    }
    if (waves == 4) hipLaunchKernelGGL((tree_fp32_kernel<D, RW, 4>), grid, dim3(256), 0, stream, p);
    if (waves == kStreamWaves) hipLaunchKernelGGL((tree_fp32_kernel<D, RW, kStreamWaves>), grid, dim3(64 * kStreamWaves), 0, stream, p);
    if (p.cut) hipLaunchKernelGGL((tree_join_ranges_kernel<T, D, kFp32Rows * RW>), join, dim3(256), 0, stream, p);
  }
}

template <int D>
static void launch_wide(const TreeParams& p, int64_t pieces, unsigned parts, hipStream_t stream) {
  const unsigned groups = (unsigned)(pieces * p.n_kv_heads);
  hipLaunchKernelGGL((tree_wide_kernel<D>), dim3(groups), dim3(256), 0, stream, p);
  // (tiles of few pieces: their workgroups would take several vectors one after another)
  if (p.cut) hipLaunchKernelGGL((tree_join_wide_kernel<D>), dim3(groups, parts), dim3(256), 0, stream, p);
}

template <typename T, int D>
static int32_t launch_tree(TreeParams& p, const TreePlan& pl, bool wide, hipStream_t stream) {
  if (!wide) {
    hipLaunchKernelGGL((tree_row_kernel<T, D>), dim3((unsigned)p.total * (unsigned)p.n_q_heads), dim3(64), 0, stream, p);
  } else {
    if constexpr (sizeof(T) == 2) {
      if (pl.wide) launch_wide<D>(p, pl.pieces, pl.join_parts, stream);
    }
    if (!pl.wide) {
      if (pl.rw == 1)
        launch_tree<T, D, 1>(p, pl.pieces, pl.waves, stream);
      else if (pl.rw == 2)
        launch_tree<T, D, 2>(p, pl.pieces, pl.waves, stream);
      else
        launch_tree<T, D, 4>(p, pl.pieces, pl.waves, stream);
    }
  }
  return hipGetLastError() == hipSuccess ? SYMPH_OK : SYMPH_ELAUNCH;
}

}  // namespace symph

using namespace symph;

extern "C" {

int64_t symph_tree_attn_workspace_bytes(const symph_kv_cache* cache, int32_t n_sessions, int32_t n_q_heads,
                                        int32_t total_new_tokens, int32_t max_new_len, int32_t max_prefix_len) {
  if (validate_cache(cache) != SYMPH_OK || n_sessions < 0 || n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0 ||
      total_new_tokens < 0 || max_new_len < 0 || max_prefix_len < 0)
    return -1;
  TreePlan pl;
  if (!plan_tree(pl, cache, n_sessions, n_q_heads, total_new_tokens, max_new_len, max_prefix_len)) return -1;
  return pl.bytes;
}

int32_t symph_tree_attn(const symph_kv_cache* cache, int32_t layer, const void* d_q, const void* d_k_new,
                        const void* d_v_new, void* d_out, const uint64_t* d_tree_mask, int32_t mask_words,
                        const int32_t* d_cu_new_lens, const int32_t* d_prefix_lens, const int32_t* d_block_table,
                        int32_t table_stride, int32_t n_sessions, int32_t n_q_heads, int32_t total_new_tokens,
                        int32_t max_new_len, int32_t max_prefix_len, float scale, void* d_workspace,
                        int64_t workspace_bytes, void* stream) {
  const int32_t rc = validate_cache(cache);
  if (rc != SYMPH_OK) return rc;
  if (layer < 0 || layer >= cache->n_layers) return SYMPH_EINVAL;
  if (n_sessions < 0 || total_new_tokens < 0 || max_new_len < 0 || max_prefix_len < 0 || table_stride < 0 ||
      workspace_bytes < 0 || mask_words < 0)
    return SYMPH_EINVAL;
  if (n_q_heads <= 0 || n_q_heads % cache->n_kv_heads != 0) return SYMPH_EINVAL;
  if (!(scale > 0.0f) || !(scale < INFINITY)) return SYMPH_EINVAL;
  if (max_new_len > total_new_tokens || (int64_t)mask_words * 64 < max_new_len || mask_words > 0x3FFFFFFF) return SYMPH_EINVAL;
  if (n_sessions == 0 || total_new_tokens == 0) return SYMPH_OK;
  if (!d_q || !d_k_new || !d_v_new || !d_out || !d_tree_mask || mask_words == 0 || !d_cu_new_lens || !d_prefix_lens)
    return SYMPH_EINVAL;
  if (max_prefix_len > 0 && (!d_block_table || table_stride == 0)) return SYMPH_EINVAL;
  if (max_prefix_len > 0 && (int64_t)table_stride * cache->block_size < max_prefix_len) return SYMPH_EINVAL;
  if (cache->head_dim != 64 && cache->head_dim != 128) return SYMPH_EUNSUPPORTED;
  if ((int64_t)total_new_tokens * n_q_heads > 0x7FFFFFFFLL) return SYMPH_EUNSUPPORTED;
  TreePlan pl;
  if (!plan_tree(pl, cache, n_sessions, n_q_heads, total_new_tokens, max_new_len, max_prefix_len)) return SYMPH_EUNSUPPORTED;
  const int eb = elem_bytes_of(cache->dtype);
  TreeParams p;
  p.k_layer = (const char*)cache->k_base + (int64_t)layer * cache->layer_stride * eb;
  p.v_layer = (const char*)cache->v_base + (int64_t)layer * cache->layer_stride * eb;
  p.block_stride = cache->block_stride;
  p.n_blocks = cache->n_blocks;
  p.block_size = cache->block_size;
  p.n_kv_heads = cache->n_kv_heads;
  p.n_q_heads = n_q_heads;
  p.q = d_q;
  p.k_new = d_k_new;
  p.v_new = d_v_new;
  p.out = d_out;
  p.mask = (const uint32_t*)d_tree_mask;
  p.mask_words = 2 * mask_words;
  p.cu_new_lens = d_cu_new_lens;
  p.prefix_lens = d_prefix_lens;
  p.table = d_block_table;
  p.table_stride = d_block_table ? table_stride : 0;
  p.n_sessions = n_sessions;
  p.total = total_new_tokens;
  p.scale = scale;
  const int64_t block_bytes = cache->block_stride * (int64_t)eb;
  p.group_bytes = grouped_rows(cache) ? (uint32_t)block_bytes : 0;
  // With 2^l >= block_size > 2^(l - 1): the factor 2^(31 + l) / block_size, rounded up, is off by less than 2^-31 of itself
  int l = 1;
  while (((int64_t)1 << l) < p.block_size) ++l;
  p.bs_magic = (uint32_t)(((uint64_t)1 << (31 + l)) / (uint64_t)p.block_size + 1);
  p.bs_more = (uint32_t)(l - 1);
  p.max_pieces = (int32_t)pl.pieces;
  p.c_min = pl.c_min;
  p.cut = pl.cut;
  p.group = n_q_heads / cache->n_kv_heads;
  const auto log2_or_neg = [](int32_t v) { return (v & (v - 1)) == 0 ? __builtin_ctz((unsigned)v) : -1; };
  p.group_shift = log2_or_neg(p.group);
  p.heads_shift = log2_or_neg(cache->n_kv_heads);
  p.aligned = pl.aligned;
  p.slots = (int32_t)std::max<int64_t>((pl.wide ? kWideSlots : kRanges) / cache->n_kv_heads, 1);
  p.parts = (float*)d_workspace;
  const uintptr_t address_bits = (uintptr_t)p.k_layer | (uintptr_t)p.v_layer | (uintptr_t)d_q | (uintptr_t)d_k_new |
                                 (uintptr_t)d_v_new | (uintptr_t)d_out | (uintptr_t)block_bytes;
  const bool wide = (address_bits & 15) == 0;
  if (!wide && !grid_takes((int64_t)total_new_tokens * n_q_heads, 64)) return SYMPH_EUNSUPPORTED;
  if (pl.bytes > 0 && (!d_workspace || workspace_bytes < pl.bytes)) return SYMPH_EWORKSPACE;
  if (pl.bytes > 0 && ((uintptr_t)d_workspace & 15) != 0) return SYMPH_EUNSUPPORTED;
  if (cache->dtype == SYMPH_BF16)
    return cache->head_dim == 64 ? launch_tree<__bf16, 64>(p, pl, wide, (hipStream_t)stream)
                                 : launch_tree<__bf16, 128>(p, pl, wide, (hipStream_t)stream);
  return cache->head_dim == 64 ? launch_tree<float, 64>(p, pl, wide, (hipStream_t)stream)
                               : launch_tree<float, 128>(p, pl, wide, (hipStream_t)stream);
}

}  // extern "C"
