// The best continuations of every session over its beams and the vocabulary.  A candidate is a token t behind a beam r; its score is
//   score(r, t) = scores[r] + x[r][t] - log sum_u exp x[r][u]
// and candidates are ordered by score, then beam, then token.  Bound by reading the logits once, which the first launch does: every
// workgroup goes over a part of a row and leaves its largest value, its sum of exponentials and its best tokens.  The second
// launch joins them session by session.  512 rows of 128256 in bf16, 131 MB: 30 us and 5 us (HBM alone 20), the vector unit 76 % busy with
// maxima, exponentials and sums, the memory idle under the workgroups' first bars and last sortings.  Four rows of 32000 in fp32: 6.3 and 3.8 us, trips to memory one after another.
#include "attn_lanes.h"

#include <algorithm>
#include <float.h>
#include <math.h>

namespace symph {

struct BeamParams {
  const char* logits;
  const float* scores;
  const int32_t* cu_rows;
  const int32_t* cu_next;
  int32_t* parents;
  int32_t* tokens;
  float* next_scores;
  float* end_scores;
  // Of each part of a row: sum of exp(x - top), that top, its best tokens (-1: no more)
  double* part_sum;     // [n_rows][parts]
  float* part_top;      // [n_rows][parts]
  float* cand_value;    // [n_rows][parts][max_next]
  int32_t* cand_token;
  float* end_logit;     // [n_rows]
  double* end_value;    // [n_rows], for sessions of many beams
  int64_t row_stride;
  int32_t n_rows, vocab, n_sessions, total_next, max_next, end_token, parts, part_tiles;
  int32_t wide;  // fp32
};

__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : fminf(x, FLT_MAX); }
__device__ __forceinline__ bool alive(float score) { return fabsf(score) <= FLT_MAX; }

// ---- the best of a list ------------------------------------------------------------------------------------------
// Values as whole numbers of the same order (zeros of both signs are equal), and back.
__device__ __forceinline__ uint32_t key_of(float x) {
  const int32_t b = __float_as_int(x + 0.0f);
  return (uint32_t)(b ^ ((b >> 31) | (int32_t)0x80000000));
}
__device__ __forceinline__ float value_of(uint32_t k) {
  return __int_as_float((int32_t)(k & 0x80000000u ? k ^ 0x80000000u : ~k));
}
__device__ __forceinline__ uint64_t key_of(double x) {
  const int64_t b = __double_as_longlong(x + 0.0);
  return (uint64_t)(b ^ ((b >> 63) | (int64_t)0x8000000000000000LL));
}

// Lanes of the mask before this one
__device__ __forceinline__ int lanes_before(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// The value of lane l ^ M.  Inside a row of 16 lanes by data-parallel moves, beyond by exchanging rows or halves.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int M>
__device__ __forceinline__ uint32_t from_lane_xor(uint32_t v) {
  static_assert(M == 1 || M == 2 || M == 3 || M == 4 || M == 7 || M == 8 || M == 15 || M == 16 || M == 31 || M == 32 || M == 63, "");
  if constexpr (M == 1) return moved<0xB1>(v);        // quad_perm:[1,0,3,2]
  if constexpr (M == 2) return moved<0x4E>(v);        // quad_perm:[2,3,0,1]
  if constexpr (M == 3) return moved<0x1B>(v);        // quad_perm:[3,2,1,0]
  if constexpr (M == 7) return moved<0x141>(v);       // row_half_mirror
  if constexpr (M == 4) return moved<0x1B>(moved<0x141>(v));
  if constexpr (M == 8) return moved<0x128>(v);       // row_ror:8
  if constexpr (M == 15) return moved<0x140>(v);      // row_mirror
  if constexpr (M == 16) {
    uint32_t x = v, y = v;  // even rows twice, odd rows twice
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(x), "+v"(y));
    return threadIdx.x & 16 ? x : y;
  }
  if constexpr (M == 32) {
    uint32_t x = v, y = v;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));
    return threadIdx.x & 32 ? x : y;
  }
  if constexpr (M == 31) return from_lane_xor<16>(from_lane_xor<15>(v));
  if constexpr (M == 63) return from_lane_xor<32>(from_lane_xor<31>(v));
  return v;
}

// An entry of WORDS words, ordered by them, the first before the others.  64 entries, one to a lane, are sorted by exchanges between
// lanes, the largest into lane 0; no two are equal but empty ones (all words 0).  The time does not depend on the values.
template <int WORDS>
struct Entry {
  uint32_t w[WORDS];
};
// (the fourth of four words comes along and does not count)
template <int WORDS>
__device__ __forceinline__ bool over(const Entry<WORDS>& a, const Entry<WORDS>& b) {
  if constexpr (WORDS == 1) return a.w[0] > b.w[0];
  const uint64_t x = (uint64_t)a.w[0] << 32 | a.w[WORDS > 1 ? 1 : 0], y = (uint64_t)b.w[0] << 32 | b.w[WORDS > 1 ? 1 : 0];
  if constexpr (WORDS == 2) return x > y;
  return x > y || (x == y && a.w[WORDS > 2 ? 2 : 0] > b.w[WORDS > 2 ? 2 : 0]);
}
// The larger of lane l's and lane l ^ M's goes to the lower of the two lanes
template <int M, int WORDS>
__device__ __forceinline__ void exchange(Entry<WORDS>& e) {
  Entry<WORDS> o;
#pragma unroll
  for (int k = 0; k < WORDS; ++k) o.w[k] = from_lane_xor<M>(e.w[k]);
  constexpr int kHigh = M & (M + 1) ? M : (M + 1) / 2;  // (the bit that tells which lane is the lower one)
  const bool lower = (threadIdx.x & kHigh) == 0, take = over(o, e) == lower;
#pragma unroll
  for (int k = 0; k < WORDS; ++k) e.w[k] = take ? o.w[k] : e.w[k];
}
template <int WORDS>
__device__ __forceinline__ void sort_rest(Entry<WORDS>& e) {  // sequences of 16 that rise and fall
  exchange<8>(e);
  exchange<4>(e);
  exchange<2>(e);
  exchange<1>(e);
}
// `runs`: runs of so many lanes (a power of two) are sorted already; `limit`: lanes from there on (a power of two) are empty
template <int WORDS>
__device__ __forceinline__ void sort64(Entry<WORDS>& e, int runs = 1, int limit = 64) {
  if (runs <= 1 && limit > 1) exchange<1>(e);
  if (runs <= 2 && limit > 2) {
    exchange<3>(e);
    exchange<1>(e);
  }
  if (runs <= 4 && limit > 4) {
    exchange<7>(e);
    exchange<2>(e);
    exchange<1>(e);
  }
  if (runs <= 8 && limit > 8) {
    exchange<15>(e);
    exchange<4>(e);
    exchange<2>(e);
    exchange<1>(e);
  }
  if (runs <= 16 && limit > 16) {
    exchange<31>(e);
    sort_rest(e);
  }
  if (runs <= 32 && limit > 32) {
    exchange<63>(e);
    exchange<16>(e);
    sort_rest(e);
  }
}
__device__ __forceinline__ int power_of_two_from(int n) { return n <= 1 ? 1 : 1 << (32 - __builtin_clz(n - 1)); }
// The 64 largest of two sorted sequences, sorted
template <int WORDS>
__device__ __forceinline__ void join64(Entry<WORDS>& e, const Entry<WORDS>& with) {
  Entry<WORDS> o;
#pragma unroll
  for (int k = 0; k < WORDS; ++k) o.w[k] = from_lane_xor<63>(with.w[k]);
  const bool take = over(o, e);
#pragma unroll
  for (int k = 0; k < WORDS; ++k) e.w[k] = take ? o.w[k] : e.w[k];
  exchange<32>(e);
  exchange<16>(e);
  sort_rest(e);
}

// ---- parts of rows -----------------------------------------------------------------------------------------------
constexpr int kValues = 32, kTile = 64 * kValues;  // a lane's values of a tile, a wave's tile

typedef unsigned int u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));  // (rows begin at any element)
typedef unsigned int u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
template <typename T>
struct Loads;
template <>
struct Loads<__bf16> {
  typedef u32x4_at2 Vec;
  static constexpr int kPer = 8;
  static __device__ __forceinline__ float at(const u32x4& v, int j) {
    return __uint_as_float(j & 1 ? v[j >> 1] & 0xFFFF0000u : v[j >> 1] << 16);
  }
};
template <>
struct Loads<float> {
  typedef u32x4_at4 Vec;
  static constexpr int kPer = 4;
  static __device__ __forceinline__ float at(const u32x4& v, int j) { return __uint_as_float(v[j]); }
};

// A lane's vectors of a whole tile that begins at `from`.  Which lane has which value follows from the index alone, not from addresses:
// equal rows have equal sums.
template <typename T>
__device__ __forceinline__ void load_tile(u32x4 (&raw)[kValues / Loads<T>::kPer], const T* from) {
  constexpr int kPer = Loads<T>::kPer;
#pragma unroll
  for (int u = 0; u < kValues / kPer; ++u)
    raw[u] = __builtin_nontemporal_load(reinterpret_cast<const typename Loads<T>::Vec*>(from + (u * 64 + (threadIdx.x & 63)) * kPer));
}

// (fmaxf would first quieten every operand; a signalling NaN comes out as a NaN here, which is looked for behind the sum)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

constexpr float kLarge = 1048576.0f;
// Entries of a wave's two queues: a lane's share of a tile where one of its values may count, and tokens that do.  A wave sorts its
// tokens in from kSortFrom on, and from kSortLast on behind its last tile; the others are sorted for all waves together.  Tiles where
// kMany lanes or more have a token that counts are looked through at once.  (The call over 512 rows of 128256 in bf16 takes 34.6 us; kMany 4
// takes 36, 24 and 48 the same, and with 90 % of the tokens masked 34.4 for 33.0; kSortFrom 32 takes 35.2, 64 the same; kSortLast 8 takes
// 35.7, in fp32 55.7 for 54.8, 48 the same.)
constexpr int kQueue = 256, kTokens = 128, kSortFrom = 48, kSortLast = 24, kMany = 12;

// exp(x - top) with the rest of log2 e: the constant's own rounding would be the same for all tokens far below the top
constexpr float kLog2e = 1.44269502e+00f, kLog2eRest = 1.92596300e-08f;
__device__ __forceinline__ float exp_below(float x, float top) {
  const float d = x - top;
  return __builtin_amdgcn_exp2f(fmaf(d, kLog2e, d * kLog2eRest));
}
// The sum of exp(x - top) over a lane's values, top being at least the largest.  One instruction in front of each
// exponential takes a tenth less of the launch than three: x log2 e - c with c = top log2 e rounded, and what c is off by taken out
// behind the sum.  What is left out is (x - top) 1.3e-8 of a term, nearly the same for all rows of a call.  Values that are too large
// for that (c would be off by more than an exponential takes) go the long way.  A lane that brings none but -infinity stays on this one, whatever
// largest value it carries from earlier tiles: its terms are 0, and c is held to where `off` is small, or 0 would be multiplied by infinity.
__device__ __forceinline__ float sum_below(const float (&x)[kValues], float top, bool large) {
  float s = 0;
  if (__ballot(large) == 0) {
    const float near = __builtin_amdgcn_fmed3f(top, -kLarge, kLarge), c = near * kLog2e, off = fmaf(near, kLog2e, -c);
#pragma unroll
    for (int v = 0; v < kValues; ++v) s += __builtin_amdgcn_exp2f(fmaf(x[v], kLog2e, -c));
    return s * __builtin_amdgcn_exp2f(-off);
  }
#pragma unroll
  for (int v = 0; v < kValues; ++v) s += exp_below(x[v], top);
  return s;
}

// Sum and maximum over a wave's lanes, every lane gets them
template <int M>
__device__ __forceinline__ double plus_xor(double v) {
  const uint64_t b = (uint64_t)__double_as_longlong(v);
  return v + __longlong_as_double((long long)((uint64_t)from_lane_xor<M>((uint32_t)(b >> 32)) << 32 | from_lane_xor<M>((uint32_t)b)));
}
__device__ __forceinline__ double wave_sum(double v) {
  return plus_xor<32>(plus_xor<16>(plus_xor<8>(plus_xor<4>(plus_xor<2>(plus_xor<1>(v))))));
}
template <int M>
__device__ __forceinline__ float max_xor(float v) {
  return max3(v, __uint_as_float(from_lane_xor<M>(__float_as_uint(v))), v);
}
__device__ __forceinline__ float wave_max(float v) {
  return max_xor<32>(max_xor<16>(max_xor<8>(max_xor<4>(max_xor<2>(max_xor<1>(v))))));
}

// Best tokens of a part of a row, its largest value and its sum: each wave has every WAVES-th tile and reads it once, a tile ahead.
// A running sum is carried to a new largest value by one factor a tile.  A token waits for the next sorting if it reaches what is
// known to be reached by as many as are wanted: at first the lanes' largest values in the waves' first tiles, then the last of the best.
// Most tiles have none or a few then, and 64 entries are sorted across lanes without a branch on values.  (A list per lane that grows by
// insertion took 1847 us for 512 rows of 128256 in bf16; one sorting per tile with tokens in it 55; as it is 30.  Loads two tiles ahead:
// 39, the registers cost a wave per SIMD.)
template <typename T, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 4) void beam_parts_kernel(const BeamParams p) {
  __shared__ int queues[WAVES][kQueue], tokens[WAVES][kTokens];
  __shared__ Entry<2> lists[WAVES][64];
  __shared__ uint32_t firsts[WAVES][64];
  // What the best of the wave that is furthest reach, and the complement of the tile up to which they were found: later ones have to pass it
  __shared__ unsigned long long shared_least;
  // Tokens that wait at the end: fewer than kSortLast of a wave whose last tile had some, fewer than kSortFrom of one whose had none
  __shared__ int waiting, rest[WAVES * kSortFrom];
  __shared__ uint32_t listed;                       // waves that have sorted some
  __shared__ float tops[WAVES];
  __shared__ double sums[WAVES];
  const int part = blockIdx.x, row = blockIdx.y, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  constexpr int kPer = Loads<T>::kPer, kVecs = kValues / kPer;
  const T* const x0 = reinterpret_cast<const T*>(p.logits) + (int64_t)row * p.row_stride;
  const int first = part * p.part_tiles, end = min(first + p.part_tiles, (p.vocab + kTile - 1) / kTile);
  u32x4 raw[kVecs];
  int tile = first + wave;
  if (tile < end && (tile + 1) * kTile <= p.vocab) load_tile<T>(raw, x0 + tile * kTile);
  if (!alive(p.scores[row])) return;  // (asked for behind the first tile: one trip to memory less)
  int* const queue = queues[wave];
  const int wanted = p.max_next;
  auto largest = [](const float (&x)[kValues]) {
    float a = max3(x[0], x[1], x[2]), b = max3(x[3], x[4], x[5]);
#pragma unroll
    for (int v = 6; v < kValues - 2; v += 4) a = max3(a, x[v], x[v + 1]), b = max3(b, x[v + 2], x[v + 3]);
    return max3(max3(a, x[kValues - 2], x[kValues - 1]), b, b);
  };
  // Candidates reach the key `least`, as at least so many values as are wanted do: to begin with, that many lanes' largest in the
  // waves' first tiles.  (One more where the end token is among them.)  0: that is not known yet.
  uint32_t least = 0;
  const int count = wanted + (p.end_token >= first * kTile && p.end_token < (first + WAVES) * kTile ? 1 : 0);
  if (threadIdx.x == 0) {
    shared_least = 0;
    waiting = 0;
    listed = 0;
  }
  // (a wave by itself does that with its first tile below; so does one whose row has no whole tile)
  if (WAVES > 1 && wanted > 0 && count <= 64 && (first + 1) * kTile <= p.vocab) {
    Entry<1> e = {0};
    if (tile < end && (tile + 1) * kTile <= p.vocab) {
      float x[kValues];
#pragma unroll
      for (int v = 0; v < kValues; ++v) x[v] = Loads<T>::at(raw[v / kPer], v % kPer);
      const float here = clean(largest(x));
      e.w[0] = here > -INFINITY ? key_of(here) : 0;
    }
    firsts[wave][lane] = e.w[0];
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) e.w[0] = max(e.w[0], firsts[w][lane]);
    sort64(e);
    least = (uint32_t)__builtin_amdgcn_readlane((int)e.w[0], count - 1);
  } else {
    __syncthreads();
  }

  if (threadIdx.x == 0 && p.end_token >= first * kTile && p.end_token < end * kTile) p.end_logit[row] = clean((float)x0[p.end_token]);

  float top = -FLT_MAX;
  double sum = 0;
  Entry<2> best = {};  // the wave's best so far, sorted: key_of the value, ~token
  int n = 0, m = 0;    // entries of the two queues
  int sorted = 0;      // tokens that were sorted in
  float bar = least ? value_of(least) : -FLT_MAX;

  // Sorts the waiting tokens in.  What is left of the tile `t` and earlier ones has to reach the last of the best, later tiles have to
  // pass it (and what other waves know), or to reach it as well while shares of earlier tiles are left in the queue (`shares`).
  auto sort_in = [&](int t, bool shares) {
    wave_sync();
#pragma unroll 1
    for (int i = lane; i - lane < m; i += 64) {
      const int token = i < m ? tokens[wave][i] : 0;
      Entry<2> e;
      e.w[0] = i < m ? key_of(clean((float)x0[token])) : 0;
      e.w[1] = i < m ? ~(uint32_t)token : 0;
      sort64(e, 1, min(power_of_two_from(m - (i - lane)), 64));
      if (__ballot(best.w[0] != 0) == 0)
        best = e;
      else
        join64(best, e);
    }
    wave_sync();
    sorted += m;
    m = 0;
    const uint32_t reached = (uint32_t)__builtin_amdgcn_readlane((int)best.w[0], wanted - 1);
    if (reached == 0) return;
    bar = fmaxf(bar, value_of(reached));
    least = max(least, reached + (shares ? 0u : 1u));
    const unsigned long long mine = (unsigned long long)reached << 32 | (uint32_t)~t;
    unsigned long long theirs = 0;
    if (lane == 0) theirs = atomicMax(&shared_least, mine);
    const uint32_t their_key = (uint32_t)__builtin_amdgcn_readfirstlane((int)(theirs >> 32));
    const int their_tile = (int)~__builtin_amdgcn_readfirstlane((int)(uint32_t)theirs);
    least = max(least, their_key + (their_key != 0 && !shares && t + WAVES > their_tile ? 1u : 0u));
  };
  // A turn looks through a tile, or again through 64 lanes' shares of earlier ones.  (Few lanes of a tile have a token that counts; to
  // look for it tile by tile took a fifth of the launch, so those lanes' values are read again, many tiles' together.)
  int again = -1;  // the queue's first entry that is to be looked at again
  while (tile < end) {
    const bool fresh = again < 0, last = tile + WAVES >= end;
    if (!fresh) wave_sync();
    const int code = fresh ? tile * 64 + lane : again + lane < n ? queue[again + lane] : -1;
    const int base = max(code >> 6, 0) * kTile, l = code & 63;
    const bool whole = base + kTile <= p.vocab;
    auto index = [&](int v) { return base + (whole ? (v / kPer * 64 + l) * kPer + v % kPer : v * 64 + l); };
    float x[kValues];
    if (whole) {
      if (!fresh) {
        u32x4 old[kVecs];
#pragma unroll
        for (int u = 0; u < kVecs; ++u) old[u] = *reinterpret_cast<const typename Loads<T>::Vec*>(x0 + index(u * kPer));
#pragma unroll
        for (int v = 0; v < kValues; ++v) x[v] = Loads<T>::at(old[v / kPer], v % kPer);
      } else {
#pragma unroll
        for (int v = 0; v < kValues; ++v) x[v] = Loads<T>::at(raw[v / kPer], v % kPer);
      }
    } else {
#pragma unroll
      for (int v = 0; v < kValues; ++v) {
        const float y = (float)x0[min(index(v), p.vocab - 1)];
        x[v] = index(v) < p.vocab ? y : -INFINITY;
      }
    }
    uint32_t open = code >= 0 ? 0xFFFFFFFFu : 0;  // values that are still to be looked at, the first in the highest bit
    bool done = !fresh && again + 64 >= n;        // with the tile, behind this turn
    if (fresh) {
      if (tile + WAVES < end && base + (WAVES + 1) * kTile <= p.vocab) load_tile<T>(raw, x0 + base + WAVES * kTile);
      float here = largest(x), above, more;
      for (bool clear = false;; clear = true) {
        above = max3(top, here, here);
        more = sum_below(x, above, here > -INFINITY && fabsf(above) > kLarge);
        if (clear || __ballot(more != more) == 0) break;
#pragma unroll
        for (int v = 0; v < kValues; ++v) x[v] = clean(x[v]);  // NaN or +infinity somewhere
        here = largest(x);
      }
      sum = sum * (double)exp_below(top, above) + (double)more;
      top = above;
      bar = least ? value_of(least) : -FLT_MAX;
      if (least == 0 && wanted > 0 && wanted < 64) {
        // as many lanes (and one that may have the end token) as are wanted reach the last of the lanes' largest that count
        Entry<1> e = {here > -INFINITY ? key_of(here) : 0};
        sort64(e);
        const uint32_t t = (uint32_t)__builtin_amdgcn_readlane((int)e.w[0], wanted);
        if (t) bar = value_of(t);
      }
      const uint64_t mask = wanted > 0 ? __ballot(here >= bar) : 0;
      const bool at_once = mask != 0 && (last || least == 0 || __popcll(mask) >= kMany);
      if (mask != 0 && !at_once) {
        if (mask >> lane & 1) queue[n + lanes_before(mask)] = code;
        n += __popcll(mask);
      }
      done = n == 0 || !(last || n + 64 > kQueue);
      if (!at_once) {
        if (done)
          tile += WAVES;
        else
          again = 0;
        continue;
      }
    }
    if (p.end_token >= base && p.end_token < base + kTile) {
      const int at = p.end_token - base, v = whole ? at / (64 * kPer) * kPer + at % kPer : at >> 6;
      if ((whole ? at / kPer : at) % 64 == l) open &= ~(0x80000000u >> v);
    }
    for (bool left = true; left;) {
      uint32_t hits = 0;
#pragma unroll
      for (int v = 0; v < kValues; ++v) hits = hits + hits + (x[v] >= bar ? 1 : 0);
      hits &= open;
      for (uint64_t mask; (mask = __ballot(hits != 0)) != 0 && m + 64 <= kTokens;) {
        if (hits) {  // the value with the highest index first
          const int bit = __builtin_ctz(hits);
          tokens[wave][m + lanes_before(mask)] = index(kValues - 1 - bit);
          hits &= hits - 1;
          open ^= 1u << bit;
        }
        m += __popcll(mask);
      }
      left = __ballot(hits != 0) != 0;
      if (left || (done && m >= (last ? kSortLast : kSortFrom)) || (least == 0 && sorted + m >= wanted && !last)) sort_in(tile, fresh && done && n > 0);
    }
    if (!fresh) again = done ? -1 : again + 64;
    if (!fresh && done) n = 0;
    if (done)
      tile += WAVES;
    else if (fresh)
      again = 0;
  }
  // The wave's sum over its lanes; its tokens that wait join the others' in any order
  const float high = wave_max(top);
  sum = wave_sum(sum * (double)exp_below(top, high));
  wave_sync();
  int at = 0;
  if (lane == 0) {
    tops[wave] = high;
    sums[wave] = sum;
    if (m > 0) at = atomicAdd(&waiting, m);
  }
  at = __builtin_amdgcn_readfirstlane(at);
  if (lane < m) rest[at + lane] = tokens[wave][lane];
  if (wave > 0 && __ballot(best.w[0] != 0) != 0) {
    lists[wave][lane] = best;
    if (lane == 0) atomicOr(&listed, 1u << wave);
  }
  __syncthreads();
  if (wave != 0) return;
  const int64_t place = (int64_t)row * p.parts + part;
  {
    const bool in = lane < WAVES;
    const float each = in ? tops[lane] : -FLT_MAX, all = wave_max(each);
    const double whole = wave_sum(in ? sums[lane] * (double)exp_below(each, all) : 0.0);
    if (lane == 0) {
      p.part_sum[place] = whole;
      p.part_top[place] = all;
    }
  }
  if (wanted == 0) return;
  const int total = waiting;
#pragma unroll 1
  for (int i = lane; i - lane < total; i += 64) {
    const int token = i < total ? rest[i] : 0;
    Entry<2> e;
    e.w[0] = i < total ? key_of(clean((float)x0[token])) : 0;
    e.w[1] = i < total ? ~(uint32_t)token : 0;
    sort64(e, 1, min(power_of_two_from(total - (i - lane)), 64));
    if (__ballot(best.w[0] != 0) == 0)
      best = e;
    else
      join64(best, e);
  }
#pragma unroll 1
  for (uint32_t left = __builtin_amdgcn_readfirstlane((int)listed); left != 0; left &= left - 1) join64(best, lists[__builtin_ctz(left)][lane]);
  if (lane < wanted) {
    p.cand_value[place * wanted + lane] = value_of(best.w[0]);
    p.cand_token[place * wanted + lane] = best.w[0] ? (int32_t)~best.w[1] : -1;
  }
}

// ---- sessions ----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float logit_at(const BeamParams& p, int row, int token) {
  const int64_t at = (int64_t)row * p.row_stride + token;
  return clean(p.wide ? reinterpret_cast<const float*>(p.logits)[at] : (float)reinterpret_cast<const __bf16*>(p.logits)[at]);
}

constexpr int kSessionWaves = 16, kRows = 256;  // kRows: rows of a session whose end scores stay in LDS

// A workgroup per session, a wave per row.  A row's best are sorted by logit and token, which is the order of their scores as well (far
// from the sum's logarithm, where 64 bits do not tell scores apart, it is the logits that count); rows are then joined by score, row
// and place in the row.  A chain of trips to memory: 64 sessions of 8 rows 5 us, 7 of 2 to 24 rows of four parts 10 to 12.  (A first bar from
// the rows' largest, so that fewer entries are sorted: 17.6, the bar has to be agreed on first.)
__global__ __launch_bounds__(64 * kSessionWaves) void beam_sessions_kernel(const BeamParams p) {
  __shared__ Entry<4> lists[kSessionWaves][64];
  __shared__ double end_near[kRows];
  __shared__ float end_logit_near[kRows];
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(tid >> 6));
  const int r0 = min(max(p.cu_rows[s], 0), p.n_rows), r1 = max(min(p.cu_rows[s + 1], p.n_rows), r0);
  const int n0 = min(max(p.cu_next[s], 0), p.total_next), n1 = max(min(p.cu_next[s + 1], p.total_next), n0);
  const int width = min(n1 - n0, p.max_next);

  struct Asked {
    float cum, last, top, x;
    double sum;
    int token;
  };
  // A part's best are sorted: 2^n lanes to a part
  const int run = power_of_two_from(p.max_next), row_limit = min(power_of_two_from(p.parts * run), 64);
  const int per_batch = width > 0 ? 64 / run : 1;
  auto candidate = [&](int r, int first, float* x, int* token) {  // of the parts from `first` on
    const int part = first + lane / run, place = lane & (run - 1);
    const bool in = width > 0 && part < p.parts && place < p.max_next;
    const int64_t at = ((int64_t)r * p.parts + part) * p.max_next + place;
    *x = in ? p.cand_value[at] : 0;
    *token = in ? p.cand_token[at] : -1;
  };
  auto ask = [&](int r) {  // (of a row that is not alive this may be anything)
    Asked a;
    a.cum = p.scores[r];
    a.last = p.end_token >= 0 ? p.end_logit[r] : -INFINITY;
    a.top = lane < p.parts ? p.part_top[(int64_t)r * p.parts + lane] : -FLT_MAX;
    a.sum = lane < p.parts ? p.part_sum[(int64_t)r * p.parts + lane] : 0;
    candidate(r, 0, &a.x, &a.token);
    return a;
  };
  // Rows are taken as many together as there are waves.  Their lists meet in LDS, 64 entries' worth to a wave
  const int most = min(r1 - r0, kSessionWaves), joiners = width > 0 ? (most * run + 63) / 64 : 0;
  Entry<4> best = {};  // sorted: the score's halves, ~(row, place in it), token
  Asked next;
  if (r0 + wave < r1) next = ask(r0 + wave);
#pragma unroll 1
  for (int c0 = r0; c0 < r1; c0 += kSessionWaves) {
    const int r = c0 + wave;
    Entry<4> e = {};
    if (r < r1) {
      const Asked a = next;
      if (r + kSessionWaves < r1) next = ask(r + kSessionWaves);
      double ends = -INFINITY;
      if (alive(a.cum)) {
        float high = a.top;
        double sum = 0;
        for (int q = lane + 64; q < p.parts; q += 64) high = fmaxf(high, p.part_top[(int64_t)r * p.parts + q]);
        high = wave_max(high);
        for (int q = lane; q < p.parts; q += 64) {
          const bool first = q < 64;
          const double part = first ? a.sum : p.part_sum[(int64_t)r * p.parts + q];
          sum += part * (double)exp_below(first ? a.top : p.part_top[(int64_t)r * p.parts + q], high);
        }
        sum = wave_sum(sum);
        const double log_sum = (double)high + log(sum);
        if (a.last > -INFINITY) ends = (double)a.cum + ((double)a.last - log_sum);
        Entry<2> of_row = {};
        float x = a.x;
        int token = a.token;
#pragma unroll 1
        for (int part = 0; part < p.parts && width > 0; part += per_batch) {
          Entry<2> e;
          e.w[0] = token >= 0 ? key_of(x) : 0;
          e.w[1] = token >= 0 ? ~(uint32_t)token : 0;
          if (part + per_batch < p.parts) candidate(r, part + per_batch, &x, &token);
          sort64(e, run, row_limit);
          if (part == 0)
            of_row = e;
          else
            join64(of_row, e);
        }
        const bool there = lane < width && of_row.w[0] != 0;
        const uint64_t key = key_of((double)a.cum + ((double)value_of(of_row.w[0]) - log_sum));
        e.w[0] = there ? (uint32_t)(key >> 32) : 0;
        e.w[1] = there ? (uint32_t)key : 0;
        e.w[2] = there ? ~(uint32_t)((r - r0) * 64 + lane) : 0;
        e.w[3] = ~of_row.w[1];
      }
      if (lane == 0) {
        const bool near = r - r0 < kRows;
        (near ? end_near[r - r0] : p.end_value[r]) = ends;
        if (near) end_logit_near[r - r0] = a.last;
      }
    }
    if (lane < run) lists[wave][lane] = e;
    __syncthreads();
    if (wave < joiners) {
      const int from = wave * per_batch + lane / run;
      Entry<4> o = {};
      if (from < min(r1 - c0, kSessionWaves)) o = lists[from][lane & (run - 1)];
      sort64(o, run, min(power_of_two_from(most * run), 64));
      if (c0 == r0)
        best = o;
      else
        join64(best, o);
    }
    __syncthreads();
  }
  // Half of the joiners take what the other half has, and so on
#pragma unroll 1
  for (int half = power_of_two_from(joiners) / 2; half > 0; half >>= 1) {
    if (wave >= half && wave < min(2 * half, joiners)) lists[wave][lane] = best;
    __syncthreads();
    if (wave < half && wave + half < joiners) join64(best, lists[wave + half][lane]);
  }
  if (wave == 0) {
    lists[0][lane] = best;
    const uint64_t key = (uint64_t)best.w[0] << 32 | best.w[1];
    if (lane < width) {
      const bool there = key != 0;
      const double score = __longlong_as_double((long long)(key >> 63 ? key ^ 0x8000000000000000ull : ~key));
      p.parents[n0 + lane] = there ? r0 + (int)(~best.w[2] >> 6) : -1;
      p.tokens[n0 + lane] = there ? (int)best.w[3] : -1;
      p.next_scores[n0 + lane] = there ? (float)score : -INFINITY;
    }
  }
  for (int k = max(width, 0) + tid; k < n1 - n0; k += 64 * kSessionWaves) {
    p.parents[n0 + k] = -1;
    p.tokens[n0 + k] = -1;
    p.next_scores[n0 + k] = -INFINITY;
  }
  if (!p.end_scores) return;
  __syncthreads();
  // A wave per row: how many of the chosen, and how many other rows' ends, come before its end
  auto end_of = [&](int r) { return r - r0 < kRows ? end_near[r - r0] : p.end_value[r]; };
  for (int r = r0 + wave; r < r1; r += kSessionWaves) {
    const double mine = end_of(r);
    bool counts = mine > -INFINITY;
    if (counts) {
      const uint64_t key = key_of(mine);
      bool before = false;
      if (lane < width) {
        const Entry<4> e = lists[0][lane];
        const uint64_t other = (uint64_t)e.w[0] << 32 | e.w[1];
        const int row = r0 + (int)(~e.w[2] >> 6);
        before = other > key || (other == key && row < r);
        if (other == key && row == r) {
          const float x = r - r0 < kRows ? end_logit_near[r - r0] : p.end_logit[r], y = logit_at(p, r, (int)e.w[3]);
          before = y > x || (y == x && (int)e.w[3] < p.end_token);
        }
      }
      int place = __popcll(__ballot(before));
      for (int q0 = r0; q0 < r1 && place < width; q0 += 64) {
        const double other = q0 + lane < r1 ? end_of(q0 + lane) : -INFINITY;
        place += __popcll(__ballot(other > mine || (other == mine && q0 + lane < r)));
      }
      counts = place < width;
    }
    if (lane == 0) p.end_scores[r] = counts ? (float)mine : -INFINITY;
  }
}

// How rows are cut: into as many waves as there are places for (four to a SIMD; half as many: 39.6 against 36.3 us for 512 rows of
// 128256 in bf16), a wave having a tile at least.  Up to eight waves of a row share a workgroup: what they know of each other's first
// tiles keeps the lists short, and few parts keep the second launch short (four at most: 11.9 against 11.2 us for 32 rows, 19.0
// against 17.8 for 72 of 50001 in fp32; up to sixteen, which wait for each other: 12.7 and 17.3).
constexpr int kWavesWanted = 4096;
struct RowCut {
  int32_t parts, tiles, waves;  // parts of a row, tiles of a part, waves of a part's workgroup (1, 2, 4 or 8)
};
static RowCut cut_rows(int32_t n_rows, int32_t vocab) {
  const int64_t tiles = ceil_div64(vocab, kTile), per_row = std::min<int64_t>(tiles, std::max(kWavesWanted / std::max(n_rows, 1), 1));
  RowCut c;
  c.waves = per_row <= 1 ? 1 : per_row <= 2 ? 2 : per_row <= 4 ? 4 : 8;
  c.tiles = (int32_t)ceil_div64(tiles, ceil_div64(per_row, c.waves));
  c.parts = (int32_t)ceil_div64(tiles, c.tiles);
  return c;
}
template <typename T>
static void launch_parts(const BeamParams& p, const RowCut& cut, hipStream_t stream) {
  const dim3 grid((unsigned)cut.parts, (unsigned)p.n_rows), threads(64 * cut.waves);
  if (cut.waves == 1)
    hipLaunchKernelGGL((beam_parts_kernel<T, 1>), grid, threads, 0, stream, p);
  else if (cut.waves == 2)
    hipLaunchKernelGGL((beam_parts_kernel<T, 2>), grid, threads, 0, stream, p);
  else if (cut.waves == 4)
    hipLaunchKernelGGL((beam_parts_kernel<T, 4>), grid, threads, 0, stream, p);
  else
    hipLaunchKernelGGL((beam_parts_kernel<T, 8>), grid, threads, 0, stream, p);
}
static int64_t round256(int64_t n) { return (n + 255) & ~(int64_t)255; }

}  // namespace symph

using namespace symph;

extern "C" {

int64_t symph_beam_select_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t max_next) {
  if (n_rows < 0 || vocab <= 0 || max_next < 0 || max_next > SYMPH_BEAM_MAX) return SYMPH_EINVAL;
  const int64_t parts = (int64_t)n_rows * cut_rows(n_rows, vocab).parts;
  return round256((int64_t)n_rows * 4) + round256((int64_t)n_rows * 8) + round256(parts * 8) + round256(parts * 4) + 2 * round256(parts * max_next * 4);
}

int32_t symph_beam_select(const void* d_logits, int64_t row_stride, int32_t dtype, int32_t n_rows, int32_t vocab,
                          const float* d_scores, const int32_t* d_cu_rows, const int32_t* d_cu_next, int32_t n_sessions,
                          int32_t total_next, int32_t max_next, int32_t end_token, int32_t* d_parents, int32_t* d_tokens,
                          float* d_next_scores, float* d_end_scores, void* d_workspace, int64_t workspace_bytes, void* stream) {
  if (n_rows < 0 || vocab <= 0 || row_stride < vocab || n_sessions < 0 || total_next < 0 || max_next < 0 || workspace_bytes < 0)
    return SYMPH_EINVAL;
  if (end_token >= vocab) return SYMPH_EINVAL;
  if (elem_bytes_of(dtype) == 0 || max_next > SYMPH_BEAM_MAX) return SYMPH_EUNSUPPORTED;
  if (n_sessions == 0) return SYMPH_OK;
  if (!d_cu_rows || !d_cu_next || (n_rows > 0 && (!d_logits || !d_scores))) return SYMPH_EINVAL;
  if (total_next > 0 && (!d_parents || !d_tokens || !d_next_scores)) return SYMPH_EINVAL;
  if (d_next_scores && d_next_scores == d_scores) return SYMPH_EINVAL;
  // (a grid's second axis takes 65535 workgroups; tiles are counted in 32 bits)
  if (n_rows > 65535 || vocab > 0x7FFFFFFF - 16 * kTile || !grid_takes(n_sessions, 64 * kSessionWaves)) return SYMPH_EUNSUPPORTED;
  if (workspace_bytes < symph_beam_select_workspace_bytes(n_rows, vocab, max_next) || (!d_workspace && n_rows > 0))
    return SYMPH_EWORKSPACE;
  if (n_rows > 0 && ((uintptr_t)d_workspace & 255) != 0) return SYMPH_EUNSUPPORTED;
  const RowCut cut = cut_rows(n_rows, vocab);
  const int64_t parts = (int64_t)n_rows * cut.parts;
  BeamParams p;
  p.logits = (const char*)d_logits;
  p.scores = d_scores;
  p.cu_rows = d_cu_rows;
  p.cu_next = d_cu_next;
  p.parents = d_parents;
  p.tokens = d_tokens;
  p.next_scores = d_next_scores;
  p.end_scores = d_end_scores;
  char* at = (char*)d_workspace;
  auto take = [&](int64_t bytes) {
    char* const here = at;
    at += round256(bytes);
    return here;
  };
  p.end_logit = (float*)take((int64_t)n_rows * 4);
  p.end_value = (double*)take((int64_t)n_rows * 8);
  p.part_sum = (double*)take(parts * 8);
  p.part_top = (float*)take(parts * 4);
  p.cand_value = (float*)take(parts * max_next * 4);
  p.cand_token = (int32_t*)take(parts * max_next * 4);
  p.row_stride = row_stride;
  p.n_rows = n_rows;
  p.vocab = vocab;
  p.n_sessions = n_sessions;
  p.total_next = total_next;
  p.max_next = max_next;
  p.end_token = end_token;
  p.parts = cut.parts;
  p.part_tiles = cut.tiles;
  p.wide = dtype == SYMPH_FP32;
  hipStream_t st = (hipStream_t)stream;
  if (n_rows > 0 && dtype == SYMPH_BF16) launch_parts<__bf16>(p, cut, st);
  if (n_rows > 0 && dtype == SYMPH_FP32) launch_parts<float>(p, cut, st);
  hipLaunchKernelGGL(beam_sessions_kernel, dim3((unsigned)n_sessions), dim3(64 * kSessionWaves), 0, st, p);
  return hipGetLastError() == hipSuccess ? SYMPH_OK : SYMPH_ELAUNCH;
}

}  // extern "C"
