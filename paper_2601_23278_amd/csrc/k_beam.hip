// A step of beam search: the best continuations of every request's beams.
//
// score(b, v) = scores[b] + (l_bv - lse_b) in 64 bits, lse = m + log(sum_v exp(l_v - m)) to 2^-34.  Within a beam the order of the scores is that of the logits, so a beam
// gives its k largest logits (ties: lower token) and its lse, and the picks come from n_beams lists of k.
//
// Two launches.  k_beam_scan reads every logit once: a row is cut into parts, one workgroup each, which leaves the part's maximum, its sum of exponentials and its
// k largest logits, sorted.  k_beam_pick puts a request's parts together.  The scan is bound by the 64-bit exponentials, 26 vector
// instructions a logit in all (counted: 2.9e7 for 512 rows of 151935): beams are compared with each other by their log-sums, and sums of fp32 exponentials (1e-7) would decide close calls by their rounding.
#include <algorithm>
#include <float.h>

#include "focus_branch.h"

namespace fk {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_any __attribute__((ext_vector_type(4), aligned(2)));      // at the address of any bf16

// Larger key: larger logit, then lower token.  0 stands for no candidate.
__device__ __forceinline__ uint64_t logit_key(float l, int token) {
  const uint32_t u = __float_as_uint(l + 0.f);         // -0 as 0
  return (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (uint32_t)~token;
}
__device__ __forceinline__ float key_logit(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_token(uint64_t key) { return (int)~(uint32_t)key; }

// exp(d) for -700 <= d <= 700, to 1.1e-12: d = n log 2 + r, |r| <= 0.347, and the polynomial of degree 8 that meets exp at nine Chebyshev nodes of that interval.
// n comes from the last bits of a sum with 1.5 * 2^52, whose neighbours lie 1 apart, and 2^n goes into the exponent's bits.
__device__ __forceinline__ double exp64(double d) {
  typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
  constexpr double unit = 6755399441055744.0;
  const double t = __builtin_fma(d, 1.4426950408889634074, unit);
  const double r = __builtin_fma(t - unit, -0.69314718055994530942, d);
  double p = 2.487623871994097e-05;
  p = __builtin_fma(p, r, 0.00019915941664891244);
  p = __builtin_fma(p, r, 0.0013888821542986098);
  p = __builtin_fma(p, r, 0.008333265963232838);
  p = __builtin_fma(p, r, 0.041666666891631156);
  p = __builtin_fma(p, r, 0.16666666891720291);
  p = __builtin_fma(p, r, 0.49999999999797123);
  p = __builtin_fma(p, r, 0.9999999999797041);
  p = __builtin_fma(p, r, 1.0);
  u32x2 w = __builtin_bit_cast(u32x2, p);
  w[1] += __builtin_bit_cast(u32x2, t)[0] << 20;
  return __builtin_bit_cast(double, w);
}
// Factor that takes a sum of exp(l - m) to one of exp(l - m_new).
__device__ __forceinline__ double rescale(float m, float m_new) {
  const double d = (double)m - (double)m_new;
  return m == m_new ? 1.0 : d < -700.0 ? 0.0 : exp64(d);
}

constexpr int kMostLists = 1024;       // of a request
struct BeamPlan {
  int parts, part;          // parts of a row and logits of a part
  double *sum;              // [rows, parts] sum of exp(l - max) over the part
  float *max;               // [rows, parts]
  uint64_t *keys;           // [rows, parts, k] descending
};
__host__ __device__ inline BeamPlan beam_plan(int n_seq, int n_beams, int vocab, int k, void *work) {
  // About 2048 workgroups, of 4096 to 65536 logits each; a request's lists (n_beams * parts) at most 1024, as far as a part may have all of a row.
  const int64_t rows = (int64_t)n_seq * n_beams;
  int64_t part = (rows * vocab / 2048 + 2047) / 2048 * 2048;
  part = part < 4096 ? 4096 : part > 65536 ? 65536 : part;
  const int64_t most = kMostLists / n_beams, least = (vocab + most - 1) / most;
  if (part < least) part = (least + 2047) / 2048 * 2048;
  BeamPlan p;
  p.parts = (int)((vocab + part - 1) / part);
  p.part = (int)part;
  if (p.parts > 1 && vocab - (p.parts - 1) * part < part / 2) {       // a short last part rules little out and would be the last to end: parts alike
    p.part = ((vocab + p.parts - 1) / p.parts + 63) / 64 * 64;        // (4 beams of 151936: 29.6 -> 16.6 us)
    p.parts = (vocab + p.part - 1) / p.part;
  }
  p.sum = (double *)work;
  p.keys = (uint64_t *)(p.sum + rows * p.parts);
  p.max = (float *)(p.keys + rows * p.parts * k);
  return p;
}
int64_t beam_groups(int n_seq, int n_beams, int vocab, int k) { return (int64_t)n_seq * n_beams * beam_plan(n_seq, n_beams, vocab, k, nullptr).parts; }
size_t beam_scratch(int n_seq, int n_beams, int vocab, int k) {
  const BeamPlan p = beam_plan(n_seq, n_beams, vocab, k, nullptr);
  return (size_t)n_seq * n_beams * p.parts * (8 + 4 + 8 * (size_t)k);
}

constexpr int kCandidates = 512;       // that a workgroup holds at a time

// Keeps the k largest of buf[0 .. n), sorted; returns how many there are.  Every key's rank is the number of larger ones (keys are different); up to 64, 4 lanes count
// for a key.
__device__ __forceinline__ int keep_largest(uint64_t *buf, int n, int k) {
  const int by = n <= 64 ? 4 : 1, at = threadIdx.x / by;
  uint64_t mine = at < n ? buf[at] : 0, other = at + 256 < n ? buf[at + 256] : 0;
  int rank = 0, rank_other = 0;
#pragma unroll 2
  for (int j = threadIdx.x % by; j < n; j += by) {
    const uint64_t x = buf[j];
    rank += x > mine;
    rank_other += x > other;
  }
  if (by == 4) {
    rank += __shfl_xor(rank, 1);
    rank += __shfl_xor(rank, 2);
  }
  __syncthreads();
  if (mine != 0 && rank < k) buf[rank] = mine;
  if (by == 1 && other != 0 && rank_other < k) buf[rank_other] = other;
  __syncthreads();
  return min(n, k);
}

// Over a wavefront, by lane shifts inside the registers (a lane exchange through LDS takes several times the instructions, and these launches wait for their
// instructions).  Lanes without a source keep their own value (max) or add nothing (sum); lane 63 ends with the whole.
template <int CTRL> __device__ __forceinline__ float shifted(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int CTRL, int ROWS> __device__ __forceinline__ double shifted_or_0(double v) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xf, false);
  return __hiloint2double(hi, lo);
}
constexpr int kRowShift = 0x110, kLane15ToNextRow = 0x142, kLane31ToNextRows = 0x143;
__device__ __forceinline__ float wavefront_max(float v) {
  v = fmaxf(v, shifted<kRowShift + 1>(v));
  v = fmaxf(v, shifted<kRowShift + 2>(v));
  v = fmaxf(v, shifted<kRowShift + 4>(v));
  v = fmaxf(v, shifted<kRowShift + 8>(v));
  v = fmaxf(v, shifted<kLane15ToNextRow>(v));
  v = fmaxf(v, shifted<kLane31ToNextRows>(v));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
__device__ __forceinline__ double wavefront_sum(double v) {
  v += shifted_or_0<kRowShift + 1, 0xf>(v);
  v += shifted_or_0<kRowShift + 2, 0xf>(v);
  v += shifted_or_0<kRowShift + 4, 0xf>(v);
  v += shifted_or_0<kRowShift + 8, 0xf>(v);
  v += shifted_or_0<kLane15ToNextRow, 0xa>(v);
  v += shifted_or_0<kLane31ToNextRows, 0xc>(v);
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 63), __builtin_amdgcn_readlane(__double2loint(v), 63));
}

template <typename T> __device__ __forceinline__ float element(const u32x4 &v, int e) {
  return sizeof(T) == 4 ? __uint_as_float(v[e]) : __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
}

template <typename T>
__global__ __launch_bounds__(256) void k_beam_scan(BeamArgs a, BeamPlan plan) {
  constexpr int EPV = 16 / sizeof(T);                // logits of a 16-byte load
  __shared__ uint64_t buf[kCandidates];
  __shared__ double sum_s[4];
  __shared__ float max_s[4], nth_s[4];
  __shared__ int count;
  const int row = blockIdx.x, part = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = a.k;
  if (a.done && a.done[row]) return;
  const int v0 = part * plan.part, v1 = min(a.vocab, v0 + plan.part);
  const T *const l = (const T *)a.logits + (size_t)row * a.ld;
  // Which thread has a logit follows from its token alone, not from the row's address, so that beams with equal logits have equal sums: 16-byte loads begin
  // wherever the row does, and what does not fill one is a logit for each of the first threads.
  const int nvec = (v1 - v0) / EPV, loose = v0 + nvec * EPV + tid;
  const u32x4_any *const vec = (const u32x4_any *)(l + v0);
  const float none = -INFINITY;
  const u32x4 nothing = sizeof(T) == 4 ? u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u} : u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u};
  const float extra = loose < v1 ? (float)l[loose] : none;
  if (tid == 0) count = 0;

  auto push = [&](float x, int token) {
    const int at = atomicAdd(&count, 1);
    if (at < kCandidates) buf[at] = logit_key(x, token);
  };
  auto fetch = [&](int i) { return i < nvec ? (u32x4)vec[i] : nothing; };
  u32x4 now = fetch(tid), next = fetch(tid + 256);
  // The sum is kept at a reference that moves only when a logit is far above it, not at the running maximum; second and at: the largest of a thread's other loads,
  // and the load that its largest logit came with.
  float m = extra == extra ? extra : none, ref = none, second = none;
  double sum = 0.0;
  bool odd = extra != extra;
  int at = -1;
#pragma unroll 1
  for (int i0 = 0; i0 < nvec; i0 += 256) {
    const u32x4 after = fetch(i0 + tid + 512);
    float top = none;
#pragma unroll
    for (int x = 0; x < EPV; ++x) {
      const float y = element<T>(now, x);
      top = fmaxf(top, y);
      odd |= y != y;
    }
    if (i0 == 0) ref = wavefront_max(top);
    second = fmaxf(second, fminf(m, top));
    at = top > m ? i0 + tid : at;
    m = fmaxf(m, top);
    if (m > ref + 500.f) {                             // exp(700) is near the end of 64 bits
      sum = ref == none ? 0.0 : sum * rescale(ref, m);
      ref = m;
    }
    // Weights below exp(-700) count as that, and so does what is no number; the end makes up for it.
    const double at_ref = ref == none ? 0.0 : (double)ref;
    double more[2] = {0.0, 0.0};
#pragma unroll
    for (int x = 0; x < EPV; ++x) more[x & 1] += exp64(__builtin_fmax((double)element<T>(now, x) - at_ref, -700.0));
    sum += more[0] + more[1];
    now = next;
    next = after;
  }
  // The part's maximum and sum.  Each of the wavefronts whose lanes all have logits has its share of k that are not below such a one of its threads' maxima, so k of
  // the part are not below the lowest of these.
  const float wave_top = wavefront_max(m);
  sum = ref == none ? 0.0 : sum * rescale(ref, wave_top);
  if (extra == extra && extra != none) sum += rescale(extra, wave_top);
  if (odd) sum = NAN;
  sum = wavefront_sum(sum);
  const int full = max(1, min(4, nvec / 64));          // (one with fewer lanes than k: nothing is ruled out)
  float left = m, nth = wave_top;
#pragma unroll 1
  for (int i = full; i < k && nth != none; i += full) {
    if (lane == __builtin_ctzll(__ballot(left == nth))) left = none;
    nth = wavefront_max(left);
  }
  if (lane == 0) {
    max_s[wave] = wave_top;
    nth_s[wave] = nth;
    sum_s[wave] = sum;
  }
  __syncthreads();
  float lim = nth_s[0];
#pragma unroll
  for (int w = 1; w < 4; ++w) lim = w < full ? fminf(lim, nth_s[w]) : lim;
  lim = fmaxf(-FLT_MAX, lim);                          // -inf is no candidate
  // The few threads that have one of the largest look at them once more: at one load, or where they have several at all of theirs.
  if (extra >= lim) push(extra, loose);
  if (m >= lim) {
#pragma unroll 1
    for (int i = second >= lim || at < 0 ? tid : at; i < nvec; i += second >= lim || at < 0 ? 256 : nvec) {
      const u32x4 v = vec[i];
      unsigned which = 0;
#pragma unroll
      for (int e = 0; e < EPV; ++e) which |= (element<T>(v, e) >= lim ? 1u : 0u) << e;
      while (which) {
        const int token = v0 + i * EPV + __builtin_ctz(which);
        which &= which - 1;
        push((float)l[token], token);
      }
    }
  }
  __syncthreads();
  const size_t o = (size_t)row * plan.parts + part;
  if (tid == 0) {
    // no more than four: each wavefront's sum at its own maximum
    const float mm = fmaxf(fmaxf(max_s[0], max_s[1]), fmaxf(max_s[2], max_s[3]));
    double all = 0.0;
#pragma unroll 1
    for (int w = 0; w < 4; ++w) all += sum_s[w] * rescale(max_s[w], mm);
    plan.sum[o] = all;
    plan.max[o] = mm;
  }
  int n = count;
  if (n > kCandidates) {
    // Too many logits that are as large (equal or sorted ones, or few in all): once more, 256 at a time, with what is not among the k largest dropped between.
    __syncthreads();
    n = 0;
    float least = -FLT_MAX;
#pragma unroll 1
    for (int s0 = v0; s0 < v1; s0 += 256) {
      if (tid == 0) count = n;
      __syncthreads();
      const int v = s0 + tid;
      const float x = v < v1 ? (float)l[v] : none;
      if (x >= least) push(x, v);
      __syncthreads();
      n = count;
      if (n > kCandidates - 256) {
        n = keep_largest(buf, n, k);
        least = nextafterf(key_logit(buf[k - 1]), INFINITY);
      }
      __syncthreads();
    }
  }
  n = keep_largest(buf, n, k);
  if (tid < k) plan.keys[o * k + tid] = tid < n ? buf[tid] : 0;
}

// Larger for larger scores; 0 for those that are not finite.
__device__ __forceinline__ uint64_t score_key(double score) {
  const uint64_t u = (uint64_t)__double_as_longlong(score + 0.0);
  return !(fabs(score) < INFINITY) ? 0 : u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double key_score(uint64_t key) { return __longlong_as_double((long long)(key >> 63 ? key & ~(1ull << 63) : ~key)); }

// A candidate of a request: larger score first, then lower beam, then larger key.
struct Candidate {
  uint64_t score, key;
  int beam;
};
__device__ __forceinline__ bool before(const Candidate &x, const Candidate &y) {
  return x.score > y.score || (x.score == y.score && (x.beam < y.beam || (x.beam == y.beam && x.key > y.key)));
}

constexpr int kPickThreads = 1024;
static_assert(kMostLists <= kPickThreads, "a thread for each list");
// One workgroup per request.  Its lists, one for each part of each beam, are sorted.  No pick lies behind the k-th best of the lists' first candidates, and those
// before it are at most k in each of k lists; a pick's place is the number of candidates before it.  Few loads that wait for each other: one request or 64, the launch
// takes what its chain of loads and barriers takes (9.7 and 11.4 us, of 152 and 32 lists a request).
__global__ __launch_bounds__(kPickThreads) void k_beam_pick(BeamArgs a, BeamPlan plan) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int q = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = a.k, beams = a.n_beams, lists = beams * plan.parts, all = lists * k;
  Candidate *const found = (Candidate *)lds;                                    // [min(lists, k) * k]
  uint64_t *const first = (uint64_t *)(found + min(lists, k) * k);              // [lists] scores of the lists' first candidates
  __shared__ double lse[kMaxBeams], base_s[kMaxBeams];
  __shared__ int done_s[kMaxBeams], count;
  __shared__ Candidate edge;
  const int row0 = q * beams;
  const uint64_t *const keys = plan.keys + (size_t)row0 * plan.parts * k;
  const uint64_t early = tid < all ? keys[tid] : 0;                             // asked for before the sums are worked out
  const float per_k = 1.f / (float)k, per_part = 1.f / (float)plan.parts;       // whole quotients: of less than 2^17, and half a step from the next
  if (tid == 0) {
    count = 0;
    edge = Candidate{0, 0, beams};
  }
#pragma unroll 1
  for (int b = wave; b < beams; b += kPickThreads / 64) {
    const size_t o = (size_t)(row0 + b) * plan.parts;
    float m = -INFINITY;
    double sum = 0.0;
#pragma unroll 1
    for (int i0 = 0; i0 < plan.parts; i0 += 64) {
      const int i = min(i0 + lane, plan.parts - 1);
      const float mi = i0 + lane < plan.parts ? plan.max[o + i] : -INFINITY;
      const double si = i0 + lane < plan.parts ? plan.sum[o + i] : 0.0;
      float top = fmaxf(m, mi);
      top = wavefront_max(top);
      sum = sum * rescale(m, top) + (si != si ? si : mi == -INFINITY ? 0.0 : si * rescale(mi, top));
      m = top;
    }
    sum = wavefront_sum(sum);
    // To whole 2^-34.  Which thread has a logit follows from its token, so rows of the same logits have the same sum and tie.  In another order the references differ, sums are up
    // to 2e-12 apart, and that is seldom the step to the next multiple (111 of 20000 shuffled rows of 4096); beams that it parts are in the order of their scores.  A sum
    // that no order changes would take some five instructions more a logit.
    const double value = __builtin_rint(((double)m + log(sum)) * 0x1p34) * 0x1p-34;
    if (lane == 0) {
      lse[b] = value;
      base_s[b] = a.scores[row0 + b];
      done_s[b] = a.done && a.done[row0 + b];
    }
  }
  __syncthreads();
  // Candidate i of all lists' candidates, list by list.  A finished beam (whose lists hold whatever was there) has its own score, once.
  auto candidate = [&](int i, uint64_t key) {
    const int list = (int)(((float)i + 0.5f) * per_k), b = (int)(((float)list + 0.5f) * per_part);
    const bool done = done_s[b] != 0;
    Candidate c;
    c.beam = b;
    c.key = done ? 0 : key;
    c.score = done ? (i == b * plan.parts * k ? score_key(base_s[b]) : 0) : key == 0 ? 0 : score_key(base_s[b] + ((double)key_logit(key) - lse[b]));
    return c;
  };
  if (lists > k) {
    // Where the k-th best list begins.
    Candidate mine{0, 0, beams};
    if (tid < lists) {
      mine = candidate(tid * k, keys[(size_t)tid * k]);
      first[tid] = mine.score;
    }
    __syncthreads();
    int rank = 0, same = 0;
#pragma unroll 4
    for (int j = 0; j < lists; ++j) {
      const uint64_t s = first[j];
      rank += s > mine.score;
      same += s == mine.score;
    }
    if (mine.score != 0 && same > 1)
#pragma unroll 1
      for (int j = 0; j < lists; ++j)
        if (first[j] == mine.score) rank += before(candidate(j * k, keys[(size_t)j * k]), mine);
    if (mine.score != 0 && rank == k - 1) edge = mine;
    __syncthreads();
  }
  const Candidate last = edge;                         // {0, 0, beams}: there are fewer
#pragma unroll 1
  for (int i = tid; i < all; i += kPickThreads) {
    const Candidate c = candidate(i, i == tid ? early : keys[i]);
    if (c.score != 0 && !before(last, c)) found[atomicAdd(&count, 1)] = c;
  }
  __syncthreads();
  const int n = count;
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += kPickThreads / 16) {  // 16 lanes count for a candidate
    const int i = i0 + tid / 16;
    const Candidate c = found[min(i, n - 1)];
    int rank = 0;
#pragma unroll 1
    for (int j = tid & 15; j < n; j += 16) rank += before(found[j], c);
    for (int x = 1; x < 16; x <<= 1) rank += __shfl_xor(rank, x);
    if (i < n && rank < k && (tid & 15) == 0) {
      const size_t o = (size_t)q * k + rank;
      a.rows[o] = row0 + c.beam;
      a.tokens[o] = done_s[c.beam] ? a.end_token : key_token(c.key);
      a.new_scores[o] = (float)key_score(c.score);
    }
  }
  for (int i = n + tid; i < k; i += kPickThreads) {
    const size_t o = (size_t)q * k + i;
    a.rows[o] = -1;
    a.tokens[o] = -1;
    a.new_scores[o] = -INFINITY;
  }
}

void beam_select(hipStream_t s, const BeamArgs &a) {
  const BeamPlan p = beam_plan(a.n_seq, a.n_beams, a.vocab, a.k, a.work);
  const dim3 grid(a.n_seq * a.n_beams, p.parts);
  a.dtype == FOCUS_F32 ? k_beam_scan<float><<<grid, 256, 0, s>>>(a, p) : k_beam_scan<bf16_t><<<grid, 256, 0, s>>>(a, p);
  const int lists = a.n_beams * p.parts;
  const size_t lds = sizeof(Candidate) * (size_t)std::min(lists, a.k) * a.k + 8 * (size_t)lists;
  if (lds > 60 * 1024) (void)hipFuncSetAttribute((const void *)k_beam_pick, hipFuncAttributeMaxDynamicSharedMemorySize, 128 * 1024);
  k_beam_pick<<<a.n_seq, kPickThreads, lds, s>>>(a, p);
}

}  // namespace fk
