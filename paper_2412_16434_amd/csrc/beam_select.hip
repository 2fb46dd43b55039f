// The best continuations of every session over its beams and the vocabulary.  A candidate is a token t behind a beam r; its score is
//   score(r, t) = scores[r] + x[r][t] - log sum_u exp x[r][u]
// and candidates are ordered by score, then beam, then token.  Bound by reading the logits once.
#include "common.h"

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
  double* log_sums;    // [n_rows]
  float* cand_value;   // [n_rows][max_next]: a row's best tokens, best first
  int32_t* cand_token; // -1: no more
  int64_t row_stride;
  int32_t n_rows, vocab, n_sessions, total_next, max_next, end_token;
};

__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : fminf(x, FLT_MAX); }
template <typename T>
__device__ __forceinline__ float value_at(const char* row, int64_t i) {
  return clean((float)reinterpret_cast<const T*>(row)[i]);
}
__device__ __forceinline__ bool alive(float score) { return fabsf(score) <= FLT_MAX; }

template <typename T>
__global__ __launch_bounds__(256) void beam_rows_kernel(const BeamParams p) {
  __shared__ float value[256];
  __shared__ int where[256];
  __shared__ double sums[256];
  const int row = blockIdx.x, tid = threadIdx.x;
  if (!alive(p.scores[row])) return;
  const char* const x = p.logits + (int64_t)row * p.row_stride * sizeof(T);
  float best = -INFINITY;
  for (int i = tid; i < p.vocab; i += 256) best = fmaxf(best, value_at<T>(x, i));
  value[tid] = best;
  __syncthreads();
  for (int h = 128; h > 0; h >>= 1) {
    if (tid < h) value[tid] = fmaxf(value[tid], value[tid + h]);
    __syncthreads();
  }
  const float top = fmaxf(value[0], -FLT_MAX);
  double sum = 0;
  for (int i = tid; i < p.vocab; i += 256) sum += (double)expf(value_at<T>(x, i) - top);
  sums[tid] = sum;
  __syncthreads();
  for (int h = 128; h > 0; h >>= 1) {
    if (tid < h) sums[tid] += sums[tid + h];
    __syncthreads();
  }
  if (tid == 0) p.log_sums[row] = (double)top + log(sums[0]);
  float last_value = INFINITY;
  int last = -1;
  for (int k = 0; k < p.max_next; ++k) {
    float v = -INFINITY;
    int at = -1;
    for (int i = tid; i < p.vocab; i += 256) {
      const float y = value_at<T>(x, i);
      if (i != p.end_token && (y < last_value || (y == last_value && i > last)) && y > v) v = y, at = i;
    }
    __syncthreads();
    value[tid] = v;
    where[tid] = at;
    __syncthreads();
    for (int h = 128; h > 0; h >>= 1) {
      if (tid < h && (value[tid + h] > value[tid] || (value[tid + h] == value[tid] && (unsigned)where[tid + h] < (unsigned)where[tid])))
        value[tid] = value[tid + h], where[tid] = where[tid + h];
      __syncthreads();
    }
    last_value = value[0];
    last = where[0];
    if (tid == 0) {
      p.cand_value[(int64_t)row * p.max_next + k] = last_value;
      p.cand_token[(int64_t)row * p.max_next + k] = last;
    }
  }
}

// A candidate, and whether one comes before another.  (Within a beam the logits decide: far from the sum's logarithm 64 bits do not
// tell their scores apart.)
struct Candidate {
  double score;
  float logit;
  int row, token;
};
__device__ __forceinline__ bool before(const Candidate& a, const Candidate& b) {
  if (a.score != b.score) return a.score > b.score;
  if (a.row != b.row) return a.row < b.row;
  return a.logit > b.logit || (a.logit == b.logit && a.token < b.token);
}

template <typename T>
__global__ __launch_bounds__(256) void beam_sessions_kernel(const BeamParams p) {
  __shared__ Candidate best[256], chosen[SYMPH_BEAM_MAX];
  const int s = blockIdx.x, tid = threadIdx.x;
  const int r0 = min(max(p.cu_rows[s], 0), p.n_rows), r1 = max(min(p.cu_rows[s + 1], p.n_rows), r0);
  const int n0 = min(max(p.cu_next[s], 0), p.total_next), n1 = max(min(p.cu_next[s + 1], p.total_next), n0);
  const int width = min(n1 - n0, p.max_next);
  const int64_t n = (int64_t)(r1 - r0) * p.max_next;
  const Candidate none{-INFINITY, -INFINITY, 0x7FFFFFFF, 0x7FFFFFFF};
  Candidate last{INFINITY, INFINITY, -1, -1};
  for (int k = 0; k < width; ++k) {
    Candidate c = none;
    for (int64_t i = tid; i < n; i += 256) {
      const int row = r0 + (int)(i / p.max_next);
      const float cum = p.scores[row];
      if (!alive(cum)) continue;
      const int64_t at = (int64_t)row * p.max_next + i % p.max_next;
      const int token = p.cand_token[at];
      if (token < 0) continue;
      const float x = p.cand_value[at];
      const Candidate y{(double)cum + ((double)x - p.log_sums[row]), x, row, token};
      if (before(last, y) && before(y, c)) c = y;
    }
    __syncthreads();
    best[tid] = c;
    __syncthreads();
    for (int h = 128; h > 0; h >>= 1) {
      if (tid < h && before(best[tid + h], best[tid])) best[tid] = best[tid + h];
      __syncthreads();
    }
    last = best[0];
    if (tid == 0) chosen[k] = last;
  }
  __syncthreads();
  for (int k = tid; k < n1 - n0; k += 256) {
    const bool there = k < width && chosen[k].row != none.row;
    p.parents[n0 + k] = there ? chosen[k].row : -1;
    p.tokens[n0 + k] = there ? chosen[k].token : -1;
    p.next_scores[n0 + k] = there ? (float)chosen[k].score : -INFINITY;
  }
  if (!p.end_scores) return;
  auto end_of = [&](int r) {
    const float cum = p.scores[r];
    if (p.end_token < 0 || !alive(cum)) return none;
    const float x = value_at<T>(p.logits + (int64_t)r * p.row_stride * sizeof(T), p.end_token);
    return x == -INFINITY ? none : Candidate{(double)cum + ((double)x - p.log_sums[r]), x, r, p.end_token};
  };
  for (int r = r0 + tid; r < r1; r += 256) {
    const Candidate y = end_of(r);
    int rank = 0;
    if (y.row != none.row) {
      for (int k = 0; k < width; ++k) rank += before(chosen[k], y);
      for (int q = r0; q < r1 && rank < width; ++q) rank += q != r && before(end_of(q), y);
    }
    p.end_scores[r] = rank < width ? (float)y.score : -INFINITY;
  }
}

static int64_t round256(int64_t n) { return (n + 255) & ~(int64_t)255; }

}  // namespace symph

using namespace symph;

extern "C" {

int64_t symph_beam_select_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t max_next) {
  if (n_rows < 0 || vocab <= 0 || max_next < 0 || max_next > SYMPH_BEAM_MAX) return SYMPH_EINVAL;
  return round256((int64_t)n_rows * 8) + 2 * round256((int64_t)n_rows * max_next * 4);
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
  if (!grid_takes(n_rows, 256) || !grid_takes(n_sessions, 256)) return SYMPH_EUNSUPPORTED;
  if (workspace_bytes < symph_beam_select_workspace_bytes(n_rows, vocab, max_next) || (!d_workspace && n_rows > 0))
    return SYMPH_EWORKSPACE;
  BeamParams p;
  p.logits = (const char*)d_logits;
  p.scores = d_scores;
  p.cu_rows = d_cu_rows;
  p.cu_next = d_cu_next;
  p.parents = d_parents;
  p.tokens = d_tokens;
  p.next_scores = d_next_scores;
  p.end_scores = d_end_scores;
  p.log_sums = (double*)d_workspace;
  p.cand_value = (float*)((char*)d_workspace + round256((int64_t)n_rows * 8));
  p.cand_token = (int32_t*)((char*)p.cand_value + round256((int64_t)n_rows * max_next * 4));
  p.row_stride = row_stride;
  p.n_rows = n_rows;
  p.vocab = vocab;
  p.n_sessions = n_sessions;
  p.total_next = total_next;
  p.max_next = max_next;
  p.end_token = end_token;
  hipStream_t st = (hipStream_t)stream;
  if (dtype == SYMPH_BF16) {
    if (n_rows > 0) hipLaunchKernelGGL(beam_rows_kernel<__bf16>, dim3((unsigned)n_rows), dim3(256), 0, st, p);
    hipLaunchKernelGGL(beam_sessions_kernel<__bf16>, dim3((unsigned)n_sessions), dim3(256), 0, st, p);
  } else {
    if (n_rows > 0) hipLaunchKernelGGL(beam_rows_kernel<float>, dim3((unsigned)n_rows), dim3(256), 0, st, p);
    hipLaunchKernelGGL(beam_sessions_kernel<float>, dim3((unsigned)n_sessions), dim3(256), 0, st, p);
  }
  return hipGetLastError() == hipSuccess ? SYMPH_OK : SYMPH_ELAUNCH;
}

}  // extern "C"
