// A step of beam search: the best continuations of every request's beams.
//
// score(b, v) = scores[b] + (l_bv - lse_b) in 64 bits.  Within a beam the order of the scores is that of the logits, so a row gives its k largest logits (ties: lower
// token) and its lse, and the requests' picks come from n_beams lists of k.
#include "focus_branch.h"

namespace fk {

template <typename T> __device__ __forceinline__ float to_f(T v) { return (float)v; }

// Larger key: larger logit, then lower token.  A logit that is not a number counts as -inf (its row has no finite score anyway); -0 as 0.
__device__ __forceinline__ uint64_t logit_key(float l, int token) {
  const uint32_t u = __float_as_uint(l != l ? -INFINITY : l + 0.f);
  return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~token;
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_token(uint64_t key) { return (int)~(uint32_t)key; }

__device__ __forceinline__ uint64_t max_over_lanes(uint64_t v) {
  for (int x = 32; x > 0; x >>= 1) {
    const uint64_t y = __shfl_xor((unsigned long long)v, x);
    v = y > v ? y : v;
  }
  return v;
}

struct BeamWork {
  double *lse;        // [rows]
  uint64_t *keys;     // [rows, k]
};
__host__ __device__ inline BeamWork beam_work(const BeamArgs &a) {
  double *lse = (double *)a.work;
  return BeamWork{lse, (uint64_t *)(lse + (size_t)a.n_seq * a.n_beams)};
}

template <typename T>
__global__ __launch_bounds__(1024) void k_beam_row(BeamArgs a) {
  __shared__ uint64_t best_s[16];
  __shared__ double sum_s[16];
  const int r = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (a.done && a.done[r]) return;
  const T *l = (const T *)a.logits + (size_t)r * a.ld;
  const BeamWork w = beam_work(a);
  uint64_t below = ~0ull;                          // the pick before
  float top = 0.f;
  for (int j = 0; j < a.k; ++j) {
    uint64_t best = 0;
    for (int v = threadIdx.x; v < a.vocab; v += 1024) {
      const uint64_t key = logit_key(to_f(l[v]), v);
      if (key < below && key > best) best = key;
    }
    best = max_over_lanes(best);
    __syncthreads();
    if (lane == 0) best_s[wave] = best;
    __syncthreads();
    for (int i = 0; i < 16; ++i) best = best_s[i] > best ? best_s[i] : best;
    if (threadIdx.x == 0) w.keys[(size_t)r * a.k + j] = best;      // 0: the vocabulary has fewer
    below = best;
    if (j == 0) top = key_logit(best);
  }
  double sum = 0.0;
  for (int v = threadIdx.x; v < a.vocab; v += 1024) sum += exp((double)to_f(l[v]) - (double)top);
  for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
  if (lane == 0) sum_s[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) sum += sum_s[i];
    w.lse[r] = (double)top + log(sum);
  }
}

// One wavefront per request: lane i holds what is left of beam i's list.
__global__ __launch_bounds__(64) void k_beam_pick(BeamArgs a) {
  const int q = blockIdx.x, i = threadIdx.x, r = q * a.n_beams + i;
  const BeamWork w = beam_work(a);
  const bool mine = i < a.n_beams, done = mine && a.done && a.done[r];
  const double base = mine ? (double)a.scores[r] : 0.0, lse = mine && !done ? w.lse[r] : 0.0;
  int next = 0;
  for (int j = 0; j < a.k; ++j) {
    double score = -INFINITY;
    uint64_t key = 0;
    if (mine && done) {
      if (next == 0) score = base;
    } else if (mine && next < a.k && (key = w.keys[(size_t)r * a.k + next]) != 0) {
      score = base + ((double)key_logit(key) - lse);
    }
    if (!(fabs(score) < INFINITY)) score = -INFINITY;
    double best = score;
    for (int x = 32; x > 0; x >>= 1) best = fmax(best, __shfl_xor(best, x));
    const uint64_t who = __ballot(score == best);
    const bool none = best == -INFINITY;
    if (!none ? i == __builtin_ctzll(who) : i == 0) {
      const size_t o = (size_t)q * a.k + j;
      a.rows[o] = none ? -1 : r;
      a.tokens[o] = none ? -1 : done ? a.end_token : key_token(key);
      a.new_scores[o] = (float)best;
      ++next;
    }
  }
}

size_t beam_scratch(int n_seq, int n_beams, int vocab, int k) { return (size_t)n_seq * n_beams * 8 * (1 + k); }

void beam_select(hipStream_t s, const BeamArgs &a) {
  const int rows = a.n_seq * a.n_beams;
  a.dtype == FOCUS_F32 ? k_beam_row<float><<<rows, 1024, 0, s>>>(a) : k_beam_row<bf16_t><<<rows, 1024, 0, s>>>(a);
  k_beam_pick<<<a.n_seq, 64, 0, s>>>(a);
}

}  // namespace fk
