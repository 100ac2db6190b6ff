// Expert router: scores, balance bias, groups, the k best experts of every row and their weights (focus_router in the header).
//
// A row's work is a chain (scores -> groups -> k picks, each of which needs the one before), a few hundred instructions on E numbers, so a
// wavefront takes a row and everything stays in its registers: lane l holds experts l P .. l P + P - 1, P = 1, 2, 4 or 8.  Neighbours in
// a lane make ties easy: the lowest expert among equals is the lowest lane's lowest element.
//
// Picks are whole numbers that have to be those of 64-bit scores.  They are found with fp32 scores, whose errors are bounded below; a row in
// which two neighbours of the picks, the last pick and anything behind it, or a kept and a dropped group are closer than that bound is done again in 64
// bits by the same code.  Equal logits with equal biases are equal in any arithmetic and need no second look.
//
// The bounds, in u = 2^-24, half an ulp (expf is off by 2 u at most, additions and divisions are rounded to nearest):
//   sigmoid   exp 2 u, 1 + exp u, quotient u: 4 u = 2.4e-7 of the score; taken as 6e-7.
//   softmax   of a logit d below the largest: d itself is rounded, d u; exp 2 u; quotient u; the sum of up to 512 terms: 7 additions in a lane and 6 across the
//             lanes, 13 u, its terms' exp 2 u and their distances, at most 4 u (the mean of d under the softmax of 512 numbers is below 4).
//             (22 + d) u = 1.31e-6 + 6e-8 d of the score; taken as 1.4e-6 + 7e-8 d.  As d exp(-d) is at most 0.37, no more than 1.35e-6 of the largest score.
//   choice    u of itself for score + bias, and as much for each comparison's own arithmetic; taken as 2e-7.
//   all       scores below the smallest normal number, 1.2e-38, have absolute errors of a few 2^-149, and an exp that overflows loses a score of 3e-39;
//             taken as 1e-37.
// They are bounds of each choice, so two whose bounds do not meet are in the order of the exact ones, and a chain of such pairs is.
//
// Bound by that chain and the launch, not by bytes (2.2 MB at 2048 rows, 0.4 us): 256 experts, 8 picks, 8 rows 6.6 us, 2048 rows without groups 7.2, 8191
// rows with 8 groups of which 4 stay 17 to 21: among so many about a dozen are done twice, and they end the launch.
#include "focus_mx.h"

namespace fk {

namespace {

constexpr int kRouteWaves = 4;       // rows of a workgroup

__device__ __forceinline__ float lane_of(float v, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); }
__device__ __forceinline__ double lane_of(double v, int l) { return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), l), __builtin_amdgcn_readlane(__double2loint(v), l)); }
__device__ __forceinline__ float exp_of(float v) { return expf(v); }
__device__ __forceinline__ double exp_of(double v) { return exp(v); }
// Over the wavefront, by lane exchanges in the vector unit: rows of 16 lanes by 1, 2, 4 and 8, then a row's last lane to the next row, then the lower
// half's to the upper; the result is in the last lane.  Six exchanges through LDS, of which every pick waits for one after the other, took ten times as
// long (a whole call of 2048 rows 10.3 us instead of 7.2).  Lanes without a source keep `other`.
template <int CTRL, int ROWS> __device__ __forceinline__ float moved(float other, float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(v), CTRL, ROWS, 0xF, false));
}
template <int CTRL, int ROWS> __device__ __forceinline__ double moved(double other, double v) {
  return __hiloint2double(__builtin_amdgcn_update_dpp(__double2hiint(other), __double2hiint(v), CTRL, ROWS, 0xF, false),
                          __builtin_amdgcn_update_dpp(__double2loint(other), __double2loint(v), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }
template <typename R> __device__ __forceinline__ R largest(R v) {
  v = larger(v, moved<0x111, 0xF>(v, v));
  v = larger(v, moved<0x112, 0xF>(v, v));
  v = larger(v, moved<0x114, 0xF>(v, v));
  v = larger(v, moved<0x118, 0xF>(v, v));
  v = larger(v, moved<0x142, 0xA>(v, v));
  v = larger(v, moved<0x143, 0xC>(v, v));
  return lane_of(v, 63);
}
template <typename R> __device__ __forceinline__ R total(R v) {
  const R none = 0;
  v += moved<0x111, 0xF>(none, v);
  v += moved<0x112, 0xF>(none, v);
  v += moved<0x114, 0xF>(none, v);
  v += moved<0x118, 0xF>(none, v);
  v += moved<0x142, 0xA>(none, v);
  v += moved<0x143, 0xC>(none, v);
  return lane_of(v, 63);
}
// LDS traffic between the lanes of one wavefront: it runs in order, only the compiler has to keep it so
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <typename R> constexpr R kLow = -(R)INFINITY;

// Picks of one row; false (R = float only): fp32 does not decide it.  idx and score of lane j < k are those of the j-th pick.  sh: LDS of this
// wavefront, 64 * P numbers and, with fp32, twice as many more.
template <typename R, int P>
__device__ __forceinline__ bool pick(const RouteArgs &a, const float (&l)[P], const float (&bias)[P], R *sh, const int32_t *forced, int &idx, R &score) {
  constexpr bool F32 = sizeof(R) == 4;
  const focus_router &r = a.router;
  const int lane = threadIdx.x & 63, E = r.n_experts, k = r.experts_per_token, G = r.n_groups, first = lane * P;
  R s[P], c[P], top_score = 1;       // no score is larger
  float top_logit = -INFINITY;
  if (r.score == FOCUS_SCORE_SIGMOID) {
#pragma unroll
    for (int i = 0; i < P; ++i) s[i] = l[i] == l[i] ? (R)1 / ((R)1 + exp_of(-(R)l[i])) : (R)0;
  } else {
#pragma unroll
    for (int i = 0; i < P; ++i) top_logit = fmaxf(top_logit, first + i < E && l[i] == l[i] ? l[i] : -INFINITY);
    top_logit = largest(top_logit);
    R sum = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      // equal to the largest: 1, also where both are infinite; a row of -inf alone has no scores
      s[i] = first + i < E && l[i] == l[i] && top_logit > -INFINITY ? (l[i] == top_logit ? (R)1 : exp_of((R)l[i] - (R)top_logit)) : (R)0;
      sum += s[i];
    }
    sum = total(sum);
#pragma unroll
    for (int i = 0; i < P; ++i) s[i] = sum > 0 ? s[i] / sum : (R)0;
    top_score = sum > 0 ? (R)1 / sum : (R)0;
  }
  if (forced) {
#pragma unroll
    for (int i = 0; i < P; ++i) sh[first + i] = s[i];
    wave_lds_order();
    if (lane < k) {
      idx = min(max(forced[lane], 0), E - 1);
      score = sh[idx];
    }
    return true;
  }
  unsigned alive = 0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    c[i] = s[i] + (R)bias[i];
    if (l[i] != l[i] || c[i] != c[i]) c[i] = kLow<R>;
    if (first + i < E) alive |= 1u << i;
  }
  if (G > 1) {
    // a group per 64 / ceil2(G) lanes: each lane looks at every such-and-such element, then the lanes' two best are merged
    const int S = E / G, step = 64 >> (32 - __clz(G - 1)), g = lane / step, sub = lane % step;
#pragma unroll
    for (int i = 0; i < P; ++i) sh[first + i] = c[i];
    wave_lds_order();
    R t1 = kLow<R>, t2 = kLow<R>;
    if (g < G)
      for (int t = sub; t < S; t += step) {
        const R v = sh[g * S + t];
        t2 = v > t1 ? t1 : (v > t2 ? v : t2);
        t1 = v > t1 ? v : t1;
      }
    for (int d = 1; d < step; d <<= 1) {
      const R o1 = __shfl_xor(t1, d), o2 = __shfl_xor(t2, d);
      const R low = o1 > t1 ? t1 : o1, high = o2 > t2 ? o2 : t2;
      t2 = low > high ? low : high;
      t1 = o1 > t1 ? o1 : t1;
    }
    const R second = r.group_top == 2 && S > 1 ? t2 : (R)0;
    R value = t1 + second;
    if (value != value) value = kLow<R>;
    int rank = 0;
    for (int o = 0; o < G; ++o) {
      const R v = lane_of(value, o * step);
      rank += v > value || (v == value && o < g);
    }
    const bool lead = sub == 0 && g < G;
    if (F32 && r.groups_kept < G) {
      // A choice is off by at most 1.4e-6 of the row's largest score (exp, sum, division) and half an ulp of itself, and a sum by half an ulp of itself:
      // ulps of the choices, which may be large and cancel.  So every group has its own bound, and every kept one has to stay above every dropped one
      // within them.  An infinite choice (no number, or an infinite bias) is infinite in any arithmetic; a sum of two finite ones that overflowed says nothing.
      const bool infinite = fabs(t1) == (R)INFINITY || fabs(second) == (R)INFINITY;
      const R off = infinite ? (R)0 : (R)3e-6 * top_score + (R)2.5e-7 * (fabs(t1) + fabs(second));
      const bool known = infinite || (off < (R)INFINITY && fabs(value) < (R)INFINITY);
      const R least = -largest(lead && rank < r.groups_kept ? (known ? off - value : (R)INFINITY) : kLow<R>);
      const R most = largest(lead && rank >= r.groups_kept ? (known ? value + off : (R)INFINITY) : kLow<R>);
      if (!(least > most)) return false;
    }
    const uint64_t kept = __ballot(lead && rank < r.groups_kept);
    const unsigned by_s = ((1u << 20) + S - 1) / S;                 // e / S = e * by_s >> 20 for e < 512
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const unsigned group = ((unsigned)(first + i) * by_s) >> 20;
      if (first + i < E && !((kept >> (group * step)) & 1)) alive &= ~(1u << i);
    }
  }
  // What fp32 may be off by in a choice c of score s and logit l (see the top); the distance from the largest logit may be infinite, the score 0 then
  auto off = [&](R c, R s, float l) {
    const float rel = r.score == FOCUS_SCORE_SIGMOID ? 6e-7f : 1.4e-6f + 7e-8f * fminf(top_logit - l, 1e30f);
    return rel * s + 2e-7f * fabsf((float)c) + 1e-37f;
  };
  const float score_off = r.score == FOCUS_SCORE_SIGMOID ? 6e-7f : 1.45e-6f * (float)top_score;      // of any score: 1.4e-6 + 0.37 * 7e-8
  // each lane's elements by falling choice, ties by the lower element; those that cannot be chosen come last
  constexpr int kNone = 0x7FFFFFFF;
  int order[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    order[i] = (alive >> i) & 1 ? first + i : kNone;
    if (!((alive >> i) & 1)) c[i] = kLow<R>;
  }
#pragma unroll
  for (int n = 0; n < P; ++n)
#pragma unroll
    for (int i = n & 1; i + 1 < P; i += 2) {
      const bool swap = c[i + 1] > c[i] || (c[i + 1] == c[i] && order[i + 1] < order[i]);
      const R hc = swap ? c[i + 1] : c[i], lc = swap ? c[i] : c[i + 1];
      const int ho = swap ? order[i + 1] : order[i], lo = swap ? order[i] : order[i + 1];
      c[i] = hc; c[i + 1] = lc; order[i] = ho; order[i + 1] = lo;
    }
  // scores, and logits and biases for the comparison of neighbours, by expert
  float *const sh_l = (float *)(sh + 64 * P), *const sh_b = sh_l + 64 * P;
  wave_lds_order();
#pragma unroll
  for (int i = 0; i < P; ++i) {
    sh[first + i] = s[i];
    if (F32) { sh_l[first + i] = l[i]; sh_b[first + i] = bias[i]; }
  }
  wave_lds_order();
  R choice = 0;
  int found = 0;
  // the next best of the wavefront: the lowest lane among equals; its expert, or -1
  auto next_best = [&](R &best) {
    best = largest(c[0]);
    const uint64_t who = __ballot(order[0] != kNone && c[0] == best);
    if (!who) return -1;
    const int w = __ffsll((unsigned long long)who) - 1, e = __builtin_amdgcn_readlane(order[0], w);
    if (lane == w) {
#pragma unroll
      for (int i = 0; i + 1 < P; ++i) { c[i] = c[i + 1]; order[i] = order[i + 1]; }
      c[P - 1] = kLow<R>;
      order[P - 1] = kNone;
    }
    return e;
  };
  for (int j = 0; j < k; ++j) {
    R best;
    const int e = next_best(best);
    if (e < 0) break;
    if (lane == j) { idx = e; choice = best; }
    found = j + 1;
  }
  if (lane < found) score = sh[idx];
  if (!F32) return true;
  // Each pick has to stay above the next, and the last above everything that was not picked, within their errors.  Experts of equal logit and bias
  // are equal, whatever the arithmetic, and ordered by their index.
  const float ml = lane < found ? sh_l[idx] : 0.f, mb = lane < found ? sh_b[idx] : 0.f;
  const R mine = off(choice, score, ml);
  const R below = __shfl_down(choice, 1), off_below = __shfl_down(mine, 1);
  const float l_below = __shfl_down(ml, 1), b_below = __shfl_down(mb, 1);
  if (__ballot(lane + 1 < found && !(ml == l_below && mb == b_below) && choice - below <= mine + off_below)) return false;
  const R end = lane_of(choice, k - 1), least = end - lane_of(mine, k - 1), next = largest(c[0]);
  // c + 2e-7 |c| grows with c, so that the largest of the rest stands for all of them where no score's error reaches across
  if (next == kLow<R> || next + 2e-7f * fabsf((float)next) + score_off + 1e-37f < least) return true;
  const int end_e = __builtin_amdgcn_readlane(idx, k - 1);
  const float end_l = lane_of(ml, k - 1), end_b = lane_of(mb, k - 1);
  bool beyond = false;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const R si = sh[first + i], ci = si + (R)bias[i];                // not a number: nothing below holds
    const bool pick = ci > end || (ci == end && first + i <= end_e);
    if (((alive >> i) & 1) && l[i] == l[i] && ci > kLow<R> && !pick && !(l[i] == end_l && bias[i] == end_b)) beyond |= !(ci + off(ci, si, l[i]) < least);
  }
  return __ballot(beyond) == 0;
}

template <typename T, int P>
__global__ __launch_bounds__(kRouteWaves * 64) void k_route(RouteArgs a) {
  __shared__ double sh[kRouteWaves][64 * P * 3 / 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.x * kRouteWaves + wave;
  const int M = a.rows.count ? min(*a.rows.count, a.rows.cap) : a.rows.cap, E = a.router.n_experts, k = a.router.experts_per_token;
  if (row >= M) return;
  const T *lg = (const T *)a.logits + (size_t)row * a.ld;
  float l[P], bias[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int e = lane * P + i;
    l[i] = e < E ? (float)lg[e] : 0.f;
    bias[i] = a.bias && e < E ? a.bias[e] : 0.f;
  }
  const int rid = a.row_map ? a.row_map[row] : row;
  const int32_t *forced = a.route_override ? a.route_override + (size_t)rid * k : nullptr;
  int idx = 0;
  float f = 0.f, sum = 0.f, weight;
  bool decided = pick<float, P>(a, l, bias, (float *)sh[wave], forced, idx, f);
  for (int j = 0; j < k; ++j) sum += lane_of(f, j);
  // scores that fp32 holds with few bits or not at all (of logits far below zero, or far below the largest) have quotients all the same
  decided = decided && !(a.router.renormalize && (sum < 1e-30f || __ballot(lane < k && f < 1.2e-38f)));
  if (decided) {
    weight = a.router.renormalize ? a.router.route_scale * f / sum : a.router.route_scale * f;
  } else {
    double d = 0.0, total = 0.0;
    pick<double, P>(a, l, bias, sh[wave], forced, idx, d);
    for (int j = 0; j < k; ++j) total += lane_of(d, j);
    weight = (float)(a.router.renormalize ? (total > 0.0 ? a.router.route_scale * d / total : 0.0) : a.router.route_scale * d);
  }
  if (lane < k) {
    a.experts[(size_t)row * k + lane] = idx;
    a.weights[(size_t)row * k + lane] = weight;
    if (a.out_experts) a.out_experts[(size_t)rid * k + lane] = idx;
    if (a.out_weights) a.out_weights[(size_t)rid * k + lane] = weight;
  }
}

template <typename T> void launch(hipStream_t s, const RouteArgs &a) {
  const int groups = (a.rows.cap + kRouteWaves - 1) / kRouteWaves, E = a.router.n_experts;
  if (E <= 64) k_route<T, 1><<<groups, kRouteWaves * 64, 0, s>>>(a);
  else if (E <= 128) k_route<T, 2><<<groups, kRouteWaves * 64, 0, s>>>(a);
  else if (E <= 256) k_route<T, 4><<<groups, kRouteWaves * 64, 0, s>>>(a);
  else k_route<T, 8><<<groups, kRouteWaves * 64, 0, s>>>(a);
}

}  // namespace

const char *check_router(const focus_router &r) {
  if (r.n_experts < 1 || r.n_experts > 512) return "n_experts must be in 1..512";
  if (r.score != FOCUS_SCORE_SOFTMAX && r.score != FOCUS_SCORE_SIGMOID) return "score must be a FOCUS_SCORE_* value";
  if (r.n_groups < 1 || r.n_groups > 64 || r.n_experts % r.n_groups) return "n_groups must be in 1..64 and divide n_experts";
  if (r.groups_kept < 1 || r.groups_kept > r.n_groups) return "groups_kept must be in 1..n_groups";
  if (r.group_top != 1 && r.group_top != 2) return "group_top must be 1 or 2";
  if (r.experts_per_token < 1 || r.experts_per_token > 32 || r.experts_per_token > r.n_experts / r.n_groups * r.groups_kept)
    return "experts_per_token must be in 1..min(32, experts of the kept groups)";
  if (r.renormalize != 0 && r.renormalize != 1) return "renormalize must be 0 or 1";
  if (!(r.route_scale > 0.f) || r.route_scale > 3.4e38f) return "route_scale must be > 0 and finite";
  return nullptr;
}

void route(hipStream_t s, const RouteArgs &a) {
  if (a.rows.cap <= 0) return;
  if (a.dtype == FOCUS_F32) launch<float>(s, a);
  else launch<bf16_t>(s, a);
}

}  // namespace fk
