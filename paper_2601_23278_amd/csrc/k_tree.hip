// Attention of drafted tokens over the paged cache, on the matrix cores.
//
// A sequence's query rows that share a key head (rows x heads of the group: its "pairs") are multiplied against one tile of cached tokens after the other, with the
// running maximum and sum of a softmax, so K and V are read once per (sequence, key head, 32 to 128 pairs) and the kernel is bound by that stream as long as pairs
// are few.  A wavefront holds 32 pairs, a workgroup 1, 2 or 4 wavefronts on the same tile.
//
// Work is a line of tiles for each key head: sequence after sequence, block of pairs after block of pairs ("unit"), every unit as many tiles as its sequence is long.
// The line is cut into equal ranges, as many as make (ranges x key heads) "pieces" for all the workgroups that the chip holds at once, so lengths need not be alike;
// the sums of a unit that a cut goes through are put together by a second, small launch in the order of the ranges.  Where they lie follows from the lengths alone.
// The heads of a range run side by side on one XCD and read the same pages at the same time: with every head's line cut for itself, 256 sequences of 512 to 4096
// tokens took 480 us instead of 441.
//
// A tile is 128 bytes of V^T rows: 64 bf16 tokens or 32 of fp32; as bytes both types are laid out alike.  Per tile and wavefront
//   S^T = K Q^T   A = K rows from LDS, B = Q in registers: a lane owns one pair, and its scores are in its own registers
//   O^T = V^T P^T  the probabilities go as they are into the B operand, V^T rows from LDS are A
// bf16: v_mfma_f32_32x32x16_bf16; lane l of the first product takes K row sigma(l % 32) (bits 2 and 3 swapped), which makes the eight scores of a lane eight
// neighbouring tokens.  fp32: v_mfma_f32_32x32x2_f32, four for each 16-byte piece; its own lane layout has four neighbouring tokens already.
// Probabilities in bf16 are rounded once (2^-8 relative), as operand of the second product; their sum is taken before.
#include <algorithm>
#include <type_traits>

#include "focus_branch.h"

namespace fk {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// s_waitcnt immediate that waits for at most n outstanding vector-memory operations and for nothing else
constexpr int vmcnt_imm(int n) { return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8); }
#define FK_LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))
#define FK_GLB_PTR(p) ((const __attribute__((address_space(1))) void *)(p))
constexpr int kNonTemporal = 2;      // cache policy of a load (NT bit)

// How a call's line of tiles is cut.
struct TreePlan {
  int nw;                  // wavefronts of a workgroup, 32 pairs each
  int ranges;              // of a head's line; workgroups: ranges * key heads
  bool cut;                // pieces end anywhere; else at the end of a unit (no room for partial sums)
  bool starts_given;       // `starts` was written by an earlier launch
  int64_t *starts;         // [n_seq + 1] first tile (cut) or unit of every sequence on a line
  int *cuts;               // [ranges, key heads, 8] of the unit that begins in a piece and goes on behind it: first row, pairs before it, its pairs, pieces of it; 0 pairs: none
  float *part_o, *part_ml; // [2 * ranges * key heads, nw * 32, D] and [.., 2]: sums of a piece's first unit, if it began before, and of its last one, if it goes on
};
constexpr int kFewSequences = 256;   // so many starts are summed up by every workgroup for itself

// A sequence's rows and tokens; its three numbers are asked for at once.
struct Sequence {
  int r0, rows, cached;
  int total;             // tokens that its row of the table has room for (below 2^31 - 64, so that tiles of tokens can be counted in 32 bits)
};
__device__ __forceinline__ Sequence sequence(const TreeArgs &a, int b) {
  const int c0 = a.cu[b], c1 = a.cu[b + 1], len = a.lens[b];
  const int64_t room = min((int64_t)a.g.stride * a.g.page_size, (int64_t)(1u << 31) - 128);
  Sequence s;
  s.r0 = max(c0, 0);
  s.rows = max(0, min(c1, a.n_rows) - s.r0);
  s.cached = max(len, 0);
  s.total = (int)min((int64_t)s.cached + s.rows, room);
  return s;
}
struct Units {
  int blocks, tiles;     // blocks of pairs, tiles of tokens
};
template <int TT>
__device__ __forceinline__ Units units_of(const TreeArgs &a, const Sequence &s, int nw) {
  const int pairs = s.rows * (a.n_q_heads / a.g.n_kv_heads);
  return Units{(pairs + nw * 32 - 1) / (nw * 32), s.rows > 0 ? (s.total + TT - 1) / TT : 0};
}
template <int TT>
__device__ __forceinline__ int64_t length_of(const TreeArgs &a, int b, const TreePlan &p) {
  const Units u = units_of<TT>(a, sequence(a, b), p.nw);
  return (int64_t)u.blocks * (p.cut ? u.tiles : 1);
}

// starts[0 .. n] by a whole wavefront; n at most kFewSequences.
template <int TT>
__device__ void sum_starts(const TreeArgs &a, const TreePlan &p, int64_t *starts) {
  constexpr int PER = kFewSequences / 64;
  const int lane = threadIdx.x & 63;
  int64_t v[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = length_of<TT>(a, min(lane * PER + i, a.n_seq - 1), p);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (lane * PER + i >= a.n_seq) v[i] = 0;
    sum += v[i];
  }
  int64_t before = sum;
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up((long long)before, o);
    if (lane >= o) before += y;
  }
  before -= sum;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int b = lane * PER + i;
    if (b <= a.n_seq) starts[b] = before;
    before += v[i];
  }
  if (lane == 63 && a.n_seq == kFewSequences) starts[kFewSequences] = before;
}
// The same by one workgroup for any number of sequences.
template <int TT>
__global__ __launch_bounds__(1024) void k_tree_starts(TreeArgs a, TreePlan p) {
  __shared__ int64_t part[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t total = 0;
  for (int b0 = 0; b0 < a.n_seq; b0 += 1024) {
    const int b = b0 + threadIdx.x;
    const int64_t v = b < a.n_seq ? length_of<TT>(a, b, p) : 0;
    int64_t x = v;
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t y = __shfl_up((long long)x, o);
      if (lane >= o) x += y;
    }
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) before += part[w];
      all += part[w];
    }
    if (b < a.n_seq) p.starts[b] = total + before + x - v;
    total += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) p.starts[a.n_seq] = total;
}
// The last b of 0 .. n - 1 with starts[b] <= at.  Up to kFewSequences a wavefront counts them, else it is looked for by halves.
__device__ __forceinline__ int find_start(const int64_t *starts, int n, int64_t at) {
  if (n <= kFewSequences) {
    int count = 0;
#pragma unroll
    for (int i = 0; i < kFewSequences / 64; ++i) {
      const int b = (threadIdx.x & 63) + i * 64;
      count += __popcll(__ballot(b < n && starts[min(b, n)] <= at));
    }
    return count - 1;
  }
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (starts[mid] <= at) lo = mid; else hi = mid;
  }
  return lo;
}
constexpr int kLeastTiles = 3;       // of a range (one request of 24 rows and 4001 tokens: 24.2 us; 1, 2, 4, 6 tiles 31, 26, 23.9, 26; 33 single fp32 tokens 35.5; 35.5, 35.5, 40, 45)
__device__ __forceinline__ int64_t range_length(const TreePlan &p, int64_t total) {
  const int64_t n = (total + p.ranges - 1) / p.ranges;
  return p.cut && n < kLeastTiles ? kLeastTiles : n < 1 ? 1 : n;
}

// Whether one of the elements of 16 bytes is an infinity or not a number, and the bytes with zeros in their place.
template <typename T> __device__ __forceinline__ bool not_finite(u32x4 v) {
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) odd |= (v[i] & 0x7f800000u) == 0x7f800000u || (sizeof(T) == 2 && (v[i] & 0x7f80u) == 0x7f80u);
  return odd;
}
template <typename T> __device__ __forceinline__ u32x4 finite_part(u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool hi = (v[i] & 0x7f800000u) == 0x7f800000u, lo = (v[i] & 0x7f80u) == 0x7f80u;
    v[i] &= sizeof(T) == 4 ? (hi ? 0u : ~0u) : (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
  }
  return v;
}
// 1 where an element of 16 bytes, without the bits that `of` lacks, is one of lo .. lo + span, else 0.  Bits of +inf, -inf and NaN are such ranges.
struct BitRange {
  unsigned of, lo, span;
};
template <typename T> __device__ __forceinline__ BitRange bits_of(int kind) {     // +inf, -inf, NaN
  constexpr unsigned inf = sizeof(T) == 2 ? 0x7f80u : 0x7f800000u, all = sizeof(T) == 2 ? 0xffffu : ~0u;
  return kind == 0 ? BitRange{all, inf, 0u} : kind == 1 ? BitRange{all, inf | (all ^ (all >> 1)), 0u} : BitRange{all >> 1, inf + 1, (all >> 1) - inf - 1};
}
template <typename T> __device__ __forceinline__ u32x4 which(u32x4 v, BitRange is) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 2) {
      const unsigned lo = ((v[i] & 0xffffu & is.of) - is.lo) <= is.span ? 0x3f80u : 0u, hi = ((v[i] >> 16 & is.of) - is.lo) <= is.span ? 0x3f800000u : 0u;
      v[i] = lo | hi;
    } else {
      v[i] = ((v[i] & is.of) - is.lo) <= is.span ? 0x3f800000u : 0u;
    }
  }
  return v;
}

// acc += A B^T of 16-byte pieces along the contracted index.
template <typename T> __device__ __forceinline__ f32x16 multiply(u32x4 a, u32x4 b, f32x16 acc);
template <> __device__ __forceinline__ f32x16 multiply<bf16_t>(u32x4 a, u32x4 b, f32x16 acc) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 multiply<float>(u32x4 a, u32x4 b, f32x16 acc) {
  const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
  return acc;
}

// Four 16-byte pieces from LDS, with their wait.  In assembly because the compiler has a read of LDS wait for every load into LDS that is under way, the next tile's too:
// that, and queries that were loaded one after the other, took 26.8 us for one request of 24 rows and 4001 tokens (24.2 so).
template <int OFFSET_0, int OFFSET_1, int OFFSET_2, int OFFSET_3>
__device__ __forceinline__ void read_4(u32x4 (&to)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3) {
  asm volatile("ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%9\n\tds_read_b128 %2, %6 offset:%10\n\tds_read_b128 %3, %7 offset:%11\n\ts_waitcnt lgkmcnt(0)"
               : "=&v"(to[0]), "=&v"(to[1]), "=&v"(to[2]), "=&v"(to[3])
               : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "n"(OFFSET_0), "n"(OFFSET_1), "n"(OFFSET_2), "n"(OFFSET_3)
               : "memory");
}

// Token of a tile, counted within 32, that register r of a product of K rows holds for lanes of half `half`.
template <typename T> __device__ __forceinline__ constexpr int token_of(int r, int half) {
  return sizeof(T) == 2 ? 16 * (r >> 3) + 8 * half + (r & 7) : 8 * (r >> 2) + 4 * half + (r & 3);
}

template <typename T> __device__ __forceinline__ void store4(T *to, f32x4 v, bool wide) {
  if (wide) {
    if (sizeof(T) == 2) *(bf16x4 *)to = bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]}; else *(f32x4 *)to = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) to[e] = (T)v[e];
  }
}

// ONE: a tile lies in one page (the page size is a multiple of the tile's tokens); else groups of 8 tokens are looked up one by one.
template <typename T, int D, int NW, bool ONE>
__global__ __launch_bounds__(NW * 64, NW == 1 && D == 128 ? 1 : 2) void k_tree(TreeArgs a, TreePlan plan) {
  constexpr int ES = sizeof(T), TT = 128 / ES, RB = D * ES, TILE = 128 * D, IPW = TILE / 1024 / NW, LPR = RB / 16;
  constexpr int KS = RB / 32, U = TT / 32, DS = D / 32, GROUPS = TT / 8;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * TILE];
  __shared__ int64_t starts_s[kFewSequences + 1];
  __shared__ int found_s[NW];
  unsigned char *const Ks = lds, *const Vs = lds + TILE;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5, col = lane & 31;
  const int H = a.g.n_kv_heads, g = a.n_q_heads / H, P = a.g.page_size;
  int range = blockIdx.x / H, h = blockIdx.x % H;
  if (plan.ranges % 8 == 0) {                          // workgroups go to the eight XCDs in turn
    range = blockIdx.x / (8 * H) * 8 + blockIdx.x % 8;
    h = blockIdx.x / 8 % H;
  }
  const int piece = range * H + h;
  const int64_t *starts = plan.starts;
  if (!plan.starts_given) {
    if (wave == 0) sum_starts<TT>(a, plan, starts_s);
    __syncthreads();
    starts = starts_s;
  }
  const int64_t total_work = starts[a.n_seq], per = range_length(plan, total_work);
  const int64_t from = per * range, end = min(from + per, total_work);
  if (plan.cut && tid == 0) plan.cuts[(size_t)piece * 8 + 2] = 0;
  if (from >= end) return;

  // K rows of 1 KB a load instruction: lane l fills the 16-byte slot l of a 1 KB block of LDS, so the swizzle against bank conflicts is applied to what it fetches.
  auto swizzle = [](int row) { return RB == 128 ? (row >> 1) & 7 : row & 15; };
  // Instruction q of a wavefront fetches K rows (V^T rows) from row0 + q * RPI (8 q) on; the bits of the two do not overlap, so a lane needs one offset for each.
  constexpr int RPI = 1024 / RB;
  const int k_row0 = wave * IPW * RPI + lane / LPR, v_row0 = wave * IPW * 8 + (lane >> 3);
  const unsigned k_lane = k_row0 * RB + (((lane % LPR) ^ swizzle(k_row0)) << 4);
  const unsigned v_chunk0 = (lane & 7) ^ ((v_row0 >> 1) & 7);
  // Where a lane reads its pieces of K (row k_tl of 32) and of V^T (row col of 32); rows 32 further on lie at the same swizzle.
  const int k_tl = ES == 2 ? (col & ~12) | (col & 4) << 1 | (col & 8) >> 1 : col;
  const unsigned k_frag = (unsigned)(uintptr_t)FK_LDS_PTR(Ks) + k_tl * RB, v_frag = (unsigned)(uintptr_t)FK_LDS_PTR(Vs) + col * 128 + ((half ^ ((col >> 1) & 7)) << 4);
  const size_t page_size = page_bytes(a.g, D, ES);
  const bool wide_q = ((uintptr_t)a.q | (uintptr_t)(a.ldq * ES)) % 16 == 0, wide_o = ((uintptr_t)a.out | (uintptr_t)(a.ldo * ES)) % 16 == 0;
  // The scale's sign goes into Q; a scale of zero makes Q zero.
  const float sc = a.scale == 0.f ? 1.f : fabsf(a.scale) * 1.4426950408889634f;      // scores in the log2 domain
  const unsigned flip = a.scale < 0.f ? (ES == 2 ? 0x80008000u : 0x80000000u) : 0u;

  // A piece is a run of tiles of one unit after the other.  The loads of a unit's first tile are asked for before the unit before it is done, so the stream of
  // tiles does not stop at its end; what that takes is worked out one unit ahead.
  struct Part {
    int b, q0, tile0, tile1, tiles, r0, rows, cached, total, pages;         // tiles 0: there is none
  };
  int64_t at = from;
  int b = __builtin_amdgcn_readfirstlane(find_start(starts, a.n_seq, at));
  // Pages.  ONE: lane i holds the page of tile first + i.  Else lane i < GROUPS holds the page of the i-th 8 tokens of a tile.  A page that is none is read as page
  // 0, and its tokens are masked.
  auto look_up = [&](int row, int tile, int tiles) {
    const unsigned t = ONE ? (unsigned)min(tile + lane, tiles - 1) * TT : (unsigned)min(tile, tiles - 1) * TT + 8 * (lane & (GROUPS - 1)), i = t / (unsigned)P;
    const int p = i < (unsigned)a.g.stride ? a.g.table[(size_t)row * a.g.stride + i] : -1;
    return p < a.g.n_pages ? p : -1;
  };
  auto next_part = [&]() {
    Part p{};
    if (at >= end) return p;
    while (starts[b + 1] <= at) ++b;
    const Sequence sq = sequence(a, b);
    const Units un = units_of<TT>(a, sq, NW);
    const int64_t in = at - starts[b];
    const int unit = __builtin_amdgcn_readfirstlane((int)(!plan.cut ? in : in < (1ll << 32) ? (unsigned)in / (unsigned)un.tiles : in / un.tiles));
    p.b = b;
    p.tiles = __builtin_amdgcn_readfirstlane(un.tiles);
    p.tile0 = plan.cut ? __builtin_amdgcn_readfirstlane((int)(in - (int64_t)unit * un.tiles)) : 0;
    p.tile1 = plan.cut ? (int)min((int64_t)p.tiles, p.tile0 + (end - at)) : p.tiles;
    at += plan.cut ? p.tile1 - p.tile0 : 1;
    p.q0 = unit * NW * 32;
    p.r0 = sq.r0;
    p.rows = sq.rows;
    p.cached = sq.cached;
    p.total = sq.total;
    p.pages = look_up(b, p.tile0, p.tiles);
    return p;
  };
  const unsigned char *const k_base = (const unsigned char *)a.g.pool + (size_t)h * P * RB, *const v_base = (const unsigned char *)a.g.pool + (size_t)(H + h) * P * RB;
  auto issue_k = [&](int tile, int pages, int first) {
    const unsigned char *base = k_base;
    if (ONE) base += (size_t)max(__builtin_amdgcn_readlane(pages, tile - first), 0) * page_size + (size_t)((unsigned)tile * TT % (unsigned)P) * RB;
#pragma unroll
    for (int q = 0; q < IPW; ++q) {
      unsigned off = (k_lane ^ (swizzle(q * RPI) << 4)) + q * 1024;
      if (!ONE) {
        const int row = k_row0 + q * RPI, place = ((unsigned)tile * TT + row) % (unsigned)P;
        base = k_base + (size_t)max(__shfl(pages, row >> 3), 0) * page_size;
        off += (place - row) * RB;
      }
      __builtin_amdgcn_global_load_lds(FK_GLB_PTR(base + off), FK_LDS_PTR(Ks + (wave * IPW + q) * 1024), 16, 0, kNonTemporal);
    }
  };
  auto issue_v = [&](int tile, int pages, int first) {
    const unsigned char *base = v_base;
    if (ONE) base += (size_t)max(__builtin_amdgcn_readlane(pages, tile - first), 0) * page_size + (size_t)((unsigned)tile * TT % (unsigned)P) * ES;
#pragma unroll
    for (int q = 0; q < IPW; ++q) {
      const unsigned chunk = v_chunk0 ^ (q * 4 & 7);
      unsigned off = (unsigned)v_row0 * (P * ES) + chunk * 16;
      if (!ONE) {
        const int t = chunk * (16 / ES);
        base = v_base + (size_t)max(__shfl(pages, t >> 3), 0) * page_size;
        off += (((unsigned)tile * TT + t) % (unsigned)P - t) * ES;
      }
      __builtin_amdgcn_global_load_lds(FK_GLB_PTR(base + (size_t)q * 8 * P * ES + off), FK_LDS_PTR(Vs + (wave * IPW + q) * 1024), 16, 0, kNonTemporal);
    }
  };
  // Bit i: the page of the tile's i-th 8 tokens is one.
  auto pages_there = [&](int tile, int pages, int first) -> unsigned {
    return ONE ? (__builtin_amdgcn_readlane(pages, tile - first) >= 0 ? (1u << GROUPS) - 1 : 0u) : (unsigned)__builtin_amdgcn_ballot_w64(pages >= 0) & ((1u << GROUPS) - 1);
  };

  Part now = next_part();
  // `pages` and `first` are those of the tile whose loads are asked for next, or that is in use; ONE false: `ahead` those of the tile after it.
  int pages = now.pages, first = now.tile0, pages_ahead = 0;
  issue_k(now.tile0, pages, first);
  issue_v(now.tile0, pages, first);
  unsigned there = pages_there(now.tile0, pages, first);
  while (now.tiles > 0) {
    const int L = now.cached, total = now.total;
    const int pair = now.q0 + wave * 32 + col;
    const bool valid = pair < now.rows * g;
    const int i_row = valid ? pair / g : 0, r = now.r0 + i_row, head = h * g + (valid ? pair % g : 0);
    // Word w of the row's set of drafted tokens.
    auto seen_word = [&](int w) -> uint64_t {
      if (a.seen) return w >= 0 && w < a.seen_words ? a.seen[(size_t)r * a.seen_words + w] : 0ull;
      const int last = i_row - 64 * w;
      return w < 0 || last < 0 ? 0ull : last >= 63 ? ~0ull : (2ull << last) - 1;
    };
    u32x4 qf[KS];
    {
      const T *qp = (const T *)a.q + (size_t)r * a.ldq + (size_t)head * D;
      // All are asked for before any is waited for; a pair that is none reads its sequence's first row.
      if (wide_q) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = *(const u32x4 *)(qp + (2 * ks + half) * (16 / ES));
      } else {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const T *const from_q = qp + (2 * ks + half) * (16 / ES);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            qf[ks][e] = ES == 2 ? (unsigned)((const uint16_t *)from_q)[2 * e] | (unsigned)((const uint16_t *)from_q)[2 * e + 1] << 16 : ((const uint32_t *)from_q)[e];
        }
      }
      const unsigned keep = valid && a.scale != 0.f ? ~0u : 0u;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int e = 0; e < 4; ++e) qf[ks][e] = (qf[ks][e] ^ flip) & keep;
    }
    const uint64_t seen0 = seen_word(0);
    const Part next = next_part();
    if (!ONE) pages_ahead = now.tile0 + 1 < now.tile1 ? look_up(now.b, now.tile0 + 1, now.tiles) : next.pages;
    f32x16 o[DS];
#pragma unroll
    for (int i = 0; i < DS; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float m = -INFINITY, l = 0.f;

    // One K buffer and one V buffer, each filled again as soon as the product that reads it is done.  Loads complete in order, so "at most IPW outstanding" means
    // that the older tile is there.  Where ONE is false the page number that look_up compares is the newest load: in every tile the wavefront waits there for all before it,
    // the next tile's K too: loads of K overlap with nothing and those of V with the first product alone.
    for (int tile = now.tile0; tile < now.tile1; ++tile) {
      const bool more = tile + 1 < now.tile1, any = more || next.tiles > 0;
      const int tile_n = more ? tile + 1 : next.tile0;
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(IPW));      // K of this tile is in LDS
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      f32x16 s[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[u][e] = 0.f;
      constexpr int AT_ONCE = 4 / U;                   // pieces of 32 bytes of D
#pragma unroll
      for (int ks = 0; ks < KS; ks += AT_ONCE) {
        unsigned at_k[AT_ONCE];
#pragma unroll
        for (int x = 0; x < AT_ONCE; ++x) at_k[x] = k_frag + (((2 * (ks + x) + half) ^ swizzle(k_tl)) << 4);
        u32x4 kf[4];
        if constexpr (U == 2)
          read_4<0, 32 * RB, 0, 32 * RB>(kf, at_k[0], at_k[0], at_k[AT_ONCE - 1], at_k[AT_ONCE - 1]);
        else
          read_4<0, 0, 0, 0>(kf, at_k[0], at_k[1 % AT_ONCE], at_k[2 % AT_ONCE], at_k[3 % AT_ONCE]);
#pragma unroll
        for (int x = 0; x < 4; ++x) s[x % U] = multiply<T>(kf[x], qf[ks + x / U], s[x % U]);
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();                    // every wavefront has read K
      const unsigned there_now = there;
      if (any) {
        if (ONE) {
          if (!more) {
            pages = next.pages;
            first = next.tile0;
          } else if (tile + 1 - first == 64) {
            pages = look_up(now.b, tile + 1, now.tiles);
            first = tile + 1;
            __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
          }
        } else {
          pages = pages_ahead;
        }
        issue_k(tile_n, pages, first);
        there = pages_there(tile_n, pages, first);
        if (!ONE && more) pages_ahead = tile + 2 < now.tile1 ? look_up(now.b, tile + 2, now.tiles) : next.pages;
      }
    // Which of the tile's tokens the pair sees: bit t, token tile * TT + t.
      const int ahead = L - tile * TT;                 // tokens of the tile that are cached ones
      const bool masked = ahead < TT || there_now != (1u << GROUPS) - 1;
      uint64_t mask = ~0ull;
      if (masked) {
        if (ahead < TT) {
          if (ahead > 0) {
            mask = ((1ull << ahead) - 1) | seen0 << ahead;
          } else {
            const int j = -ahead, w = j >> 6, by = j & 63;
            mask = w == 0 ? seen0 : seen_word(w);
            if (by) mask = mask >> by | seen_word(w + 1) << (64 - by);
          }
          const int left = total - tile * TT;
          if (left < 64) mask &= (1ull << left) - 1;
        }
#pragma unroll
        for (int i = 0; i < GROUPS; ++i)
          if (!(there_now >> i & 1)) mask &= ~(0xffull << (8 * i));
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int word = (int)((unsigned)(mask >> (32 * u)) >> ((ES == 2 ? 8 : 4) * half));      // a lane's tokens at places that the compiler knows
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int keep = __builtin_amdgcn_sbfe(word, token_of<T>(e, 0), 1);
            s[u][e] = __int_as_float((keep & __float_as_int(s[u][e])) | (~keep & (int)0xff800000));
          }
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[u][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 32)) * sc;
      const float m_new = fmaxf(m, mx), m_use = m_new == -INFINITY ? 0.f : m_new, corr = __builtin_amdgcn_exp2f(m - m_use);
      m = m_new;
      u32x4 pf[4];
      float sum = 0.f;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
#pragma unroll
        for (int e = 0; e < 16 / ES; ++e) {
          const int x = kk * (16 / ES) + e;            // register of the scores, counted through
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x >> 4][x & 15], sc, -m_use));
          sum += p;
          ((T *)&pf[kk])[e] = (T)p;
        }
      }
      l = l * corr + sum;
      if (__builtin_amdgcn_ballot_w64(corr != 1.0f) != 0) {       // a pair's maximum moved
#pragma unroll
        for (int i = 0; i < DS; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[i][e] *= corr;
      }
      if (any) __builtin_amdgcn_s_waitcnt(vmcnt_imm(IPW)); else __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));   // V is in LDS
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      auto v_piece = [&](int ds, int kk) {
        const int vr = 32 * ds + col;
        return *(const u32x4 *)(Vs + vr * 128 + (((2 * kk + half) ^ ((vr >> 1) & 7)) << 4));
      };
      if (masked) {
        // A weight of zero times what is no number would be none either.  So the product takes the finite values of a tile that not every pair sees whole; where a
        // token that exists holds others, counts of +inf, -inf and NaN among the tokens that a pair sees are added up in products of their own first.
        int found = 0;                                 // 1: values that are no numbers; 3: in tokens that exist
#pragma unroll 2
        for (int i = 0; i < IPW; ++i) {
          const int vr = (wave * IPW + i) * 8 + (lane >> 3), t0 = ((lane & 7) ^ ((vr >> 1) & 7)) * (16 / ES);
          if (not_finite<T>(*(const u32x4 *)(Vs + (wave * IPW + i) * 1024 + lane * 16))) {
            const bool exists = tile * TT + t0 < total && (there_now >> (t0 >> 3) & 1);
            found |= exists ? 3 : 1;
          }
        }
        found = (__builtin_amdgcn_ballot_w64(found & 1) != 0 ? 1 : 0) | (__builtin_amdgcn_ballot_w64(found & 2) != 0 ? 2 : 0);
        if (NW > 1) {
          if (lane == 0) found_s[wave] = found;
          __syncthreads();
#pragma unroll
          for (int w = 0; w < NW; ++w) found |= found_s[w];
        }
        found = __builtin_amdgcn_readfirstlane(found);
        if (found & 2) {
#pragma unroll 1
          for (int kind = 0; kind < 3; ++kind) {
            const float is = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
            const BitRange range = bits_of<T>(kind);
#pragma unroll
            for (int ds = 0; ds < DS; ++ds) {
              f32x16 count;
#pragma unroll
              for (int e = 0; e < 16; ++e) count[e] = 0.f;
#pragma unroll
              for (int kk = 0; kk < 4; ++kk) {
                u32x4 sees;
                const unsigned seen_bits = (unsigned)(mask >> ((2 * kk + half) * (16 / ES)));
#pragma unroll
                for (int e = 0; e < 16 / ES; ++e) ((T *)&sees)[e] = (T)(float)(int)(seen_bits >> e & 1);
                count = multiply<T>(which<T>(v_piece(ds, kk), range), sees, count);
                asm volatile("" ::: "memory");
              }
#pragma unroll
              for (int e = 0; e < 16; ++e) o[ds][e] += count[e] > 0.f ? is : 0.f;
            }
          }
          __syncthreads();                             // nobody reads the values as they were any more
        }
        if (found) {
#pragma unroll 1
          for (int i = 0; i < IPW; ++i) {
            u32x4 *const at_v = (u32x4 *)(Vs + (wave * IPW + i) * 1024 + lane * 16);
            *at_v = finite_part<T>(*at_v);
          }
          __syncthreads();
        }
      }
      auto add_rows = [&](auto rows) {                 // 32 rows of V^T
        constexpr int ds = decltype(rows)::value;
        u32x4 vf[4];
        read_4<ds * 4096, ds * 4096, ds * 4096, ds * 4096>(vf, v_frag ^ (0 << 5), v_frag ^ (1 << 5), v_frag ^ (2 << 5), v_frag ^ (3 << 5));
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) o[ds] = multiply<T>(vf[kk], pf[kk], o[ds]);
      };
      add_rows(std::integral_constant<int, 0>());
      add_rows(std::integral_constant<int, 1>());
      if constexpr (DS == 4) {
        add_rows(std::integral_constant<int, 2>());
        add_rows(std::integral_constant<int, 3>());
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_barrier();                    // every wavefront has read V
      if (any) issue_v(tile_n, pages, first);
    }

    const float l_tot = l + __shfl_xor(l, 32);
    if (now.tile0 == 0 && now.tile1 < now.tiles && tid == 0) {
      int *const c = plan.cuts + (size_t)piece * 8;
      c[0] = now.r0; c[1] = now.q0; c[2] = min(now.rows * g - now.q0, NW * 32); c[3] = (int)((now.tiles - now.tile1 + per - 1) / per) + 1;
    }
    if (now.tile0 == 0 && now.tile1 == now.tiles) {
      const float inv = l_tot == 0.f ? 0.f : 1.0f / l_tot;
      T *to = (T *)a.out + (size_t)r * a.ldo + (size_t)head * D;
#pragma unroll
      for (int ds = 0; ds < DS; ++ds)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          if (valid) store4<T>(to + 32 * ds + 8 * q4 + 4 * half, f32x4{o[ds][4 * q4], o[ds][4 * q4 + 1], o[ds][4 * q4 + 2], o[ds][4 * q4 + 3]} * inv, wide_o);
    } else {
      // Sums go out register by register, 1 KB of all lanes at a time (16 bytes of every pair at a time, 32 pairs apart, took 26 us more for 33 MB).
      const size_t slot = ((size_t)2 * piece + (now.tile0 == 0)) * NW + wave;
      float *const po = plan.part_o + slot * 32 * D + lane * 4;
#pragma unroll
      for (int ds = 0; ds < DS; ++ds)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          if (valid) *(f32x4 *)(po + (ds * 4 + q4) * 256) = f32x4{o[ds][4 * q4], o[ds][4 * q4 + 1], o[ds][4 * q4 + 2], o[ds][4 * q4 + 3]};
      if (valid && half == 0) *(float2 *)(plan.part_ml + (slot * 32 + col) * 2) = make_float2(m, l_tot);
    }
    now = next;
  }
}

// Units that a cut went through: out = sum_i o_i 2^(m_i - M) / sum_i l_i 2^(m_i - M), i over the pieces in their order.  blockIdx.x is the piece that the unit begins
// in; a wavefront takes four columns for each half of its lanes of 32 pairs, as they were written, from eight pieces at a time with a running maximum.  FAR: the four
// wavefronts of a workgroup share the pieces of such columns, for few sequences in many pieces.  The launch takes what its chain of loads takes: a record, then
// everything.
template <typename T, int D, bool FAR>
__global__ __launch_bounds__(256) void k_tree_join(TreeArgs a, TreePlan plan) {
  constexpr int LINES = D / 8, AT_ONCE = 8;
  __shared__ f32x4 num_s[FAR ? 4 : 1][64];
  __shared__ float2 den_s[FAR ? 4 : 1][64];
  const int *const rec = plan.cuts + (size_t)blockIdx.x * 8;
  const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6, id = FAR ? blockIdx.y : blockIdx.y * 4 + w, wave = id / LINES, line = id % LINES;
  const int pair = wave * 32 + (lane & 31);
  const int r0 = rec[0], q0 = rec[1], pairs = rec[2], all = rec[3], H = a.g.n_kv_heads;
  if (wave * 32 >= pairs) return;
  const int share = FAR ? (all + 3) / 4 : all, n = FAR ? min(all, (w + 1) * share) : all;
  f32x4 num = {0.f, 0.f, 0.f, 0.f};
  float den = 0.f, mm = -INFINITY;
  for (int i0 = FAR ? w * share : 0; i0 < n; i0 += AT_ONCE) {
    f32x4 v[AT_ONCE];
    float2 ml[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int i = min(i0 + j, n - 1);
      const size_t slot = ((size_t)2 * (blockIdx.x + (size_t)i * H) + (i == 0)) * plan.nw + wave;
      v[j] = *(const f32x4 *)(plan.part_o + slot * 32 * D + line * 256 + lane * 4);
      ml[j] = *(const float2 *)(plan.part_ml + (slot * 32 + (lane & 31)) * 2);
    }
    float top = mm;
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) top = fmaxf(top, ml[j].x);         // the last piece twice is no other maximum
    const float old = mm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mm - top);
    den *= old;
    num *= old;
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const bool sees = i0 + j < n && (ml[j].x != -INFINITY || ml[j].y != 0.f);       // else nothing was seen there; weights that are no numbers come through
      const float k = sees ? __builtin_amdgcn_exp2f(ml[j].x - top) : 0.f;
      den += sees ? ml[j].y * k : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] += sees ? v[j][e] * k : 0.f;
    }
    mm = top;
  }
  if (FAR) {
    num_s[w][lane] = num;
    den_s[w][lane] = make_float2(mm, den);
    __syncthreads();
    if (w != 0) return;
    float2 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = den_s[i][lane];
    const float top = fmaxf(fmaxf(x[0].x, x[1].x), fmaxf(x[2].x, x[3].x));
    num = f32x4{0.f, 0.f, 0.f, 0.f};
    den = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool sees = x[i].x != -INFINITY || x[i].y != 0.f;
      const float k = sees ? __builtin_amdgcn_exp2f(x[i].x - top) : 0.f;
      den += sees ? x[i].y * k : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] += sees ? num_s[i][lane][e] * k : 0.f;
    }
  }
  if (pair >= pairs) return;
  const int g = a.n_q_heads / H, row = r0 + (q0 + pair) / g, head = blockIdx.x % H * g + (q0 + pair) % g;
  store4<T>((T *)a.out + (size_t)row * a.ldo + (size_t)head * D + 32 * (line / 4) + 8 * (line % 4) + 4 * half, num * (den == 0.f ? 0.f : 1.0f / den),
            ((uintptr_t)a.out | (uintptr_t)(a.ldo * sizeof(T))) % 16 == 0);
}

// ---------------------------------------------------------------------------------------------
namespace {

struct Shape {
  int nw, ranges;
  bool whole;              // units are not cut
  size_t starts_bytes, cuts_bytes, bytes;
};
Shape shape_of(const TreeArgs &a) {
  const int g = a.n_q_heads / a.g.n_kv_heads, es = a.dtype == FOCUS_F32 ? 4 : 2, tt = 128 / es;
  const int64_t rows = a.max_rows > 0 ? std::min(a.max_rows, a.n_rows) : std::min((int64_t)a.n_rows, 2 * (((int64_t)a.n_rows + a.n_seq - 1) / a.n_seq)), pairs = rows * g;
  Shape s;
  s.nw = pairs <= 32 ? 1 : pairs <= 64 ? 2 : 4;
  const int64_t tokens = std::min((int64_t)a.g.stride * a.g.page_size, a.max_len > 0 ? (int64_t)a.max_len : INT64_MAX);
  const int64_t blocks = ((int64_t)a.n_rows * g + s.nw * 32 - 1) / (s.nw * 32) + a.n_seq;
  const int64_t tiles = std::min((int64_t)1 << 40, blocks) * ((tokens + tt - 1) / tt);
  const int at_once = 256 * (s.nw == 4 ? 2 : a.head_dim == 64 ? 8 : 4), most = std::max(1, at_once / a.g.n_kv_heads);
  // A short unit is not cut: one launch, and sums for the join, and the join, take 7 to 9 us more.  us whole and cut, 8 heads of 128, 8 rows: 1 sequence of 108 tokens
  // 21 and 23, of 308 23 and 21; 8 of 308 24 and 25, of 708 40 and 34; 32 (as many units as compute units) of 108 20 and 30, of 1008 44 and 48; 64 of 108 19 and 34,
  // of 1008 56 and 70.  4 heads of 64: 64 of 308 20 and 25, of 1008 42 and 44, 32 of 408 23 and 22.  fp32: 8 of 104 24 and 26, of 204 33 and 24.
  const int64_t units = (int64_t)a.n_seq * a.g.n_kv_heads * ((pairs + s.nw * 32 - 1) / (s.nw * 32));
  s.whole = (tokens + tt - 1) / tt <= (es == 4 ? 4 : units >= 256 ? 16 : units >= 32 ? 6 : 3);
  s.ranges = (int)std::max((int64_t)1, std::min((int64_t)most, s.whole ? blocks : (tiles + kLeastTiles - 1) / kLeastTiles));
  if (s.ranges >= 8) s.ranges = std::min((s.ranges + 7) / 8 * 8, most / 8 * 8 ? most / 8 * 8 : most);
  const size_t pieces = (size_t)s.ranges * a.g.n_kv_heads;
  s.starts_bytes = ((size_t)a.n_seq + 1) * 8;
  s.starts_bytes = (s.starts_bytes + 255) / 256 * 256;
  s.cuts_bytes = (pieces * 32 + 255) / 256 * 256;
  s.bytes = s.whole ? (a.n_seq > kFewSequences ? s.starts_bytes : 0) : s.starts_bytes + s.cuts_bytes + 2 * pieces * s.nw * 32 * (a.head_dim + 2) * 4;
  return s;
}

template <typename T, int D, int NW>
void launch(hipStream_t s, const TreeArgs &a, const TreePlan &p) {
  if (a.g.page_size % (128 / sizeof(T)) == 0)
    k_tree<T, D, NW, true><<<p.ranges * a.g.n_kv_heads, NW * 64, 0, s>>>(a, p);
  else
    k_tree<T, D, NW, false><<<p.ranges * a.g.n_kv_heads, NW * 64, 0, s>>>(a, p);
}
template <typename T, int D>
void run(hipStream_t s, const TreeArgs &a, const TreePlan &p) {
  if (p.starts_given) k_tree_starts<128 / sizeof(T)><<<1, 1024, 0, s>>>(a, p);
  p.nw == 1 ? launch<T, D, 1>(s, a, p) : p.nw == 2 ? launch<T, D, 2>(s, a, p) : launch<T, D, 4>(s, a, p);
  if (p.cut && p.ranges >= 8 * (int64_t)a.n_seq)
    k_tree_join<T, D, true><<<dim3(p.ranges * a.g.n_kv_heads, p.nw * (D / 8)), 256, 0, s>>>(a, p);
  else if (p.cut)
    k_tree_join<T, D, false><<<dim3(p.ranges * a.g.n_kv_heads, p.nw * (D / 8) / 4), 256, 0, s>>>(a, p);
}

}  // namespace

size_t tree_scratch(const TreeArgs &a) { return shape_of(a).bytes; }

void tree_attention(hipStream_t s, const TreeArgs &a) {
  const Shape sh = shape_of(a);
  if (a.n_seq > kFewSequences && a.scratch.bytes < sh.starts_bytes) {      // nowhere to write the starts: a launch for each few sequences
    for (int b = 0; b < a.n_seq; b += kFewSequences) {
      TreeArgs few = a;
      few.n_seq = std::min(kFewSequences, a.n_seq - b);
      few.cu += b;
      few.lens += b;
      few.g.table += (size_t)b * a.g.stride;
      few.scratch = Scratch{};
      tree_attention(s, few);
    }
    return;
  }
  TreePlan p{};
  p.nw = sh.nw;
  p.ranges = sh.ranges;
  p.starts = (int64_t *)a.scratch.ptr;
  p.cut = !sh.whole && a.scratch.bytes >= sh.bytes;
  p.starts_given = a.n_seq > kFewSequences;
  p.cuts = (int *)((char *)a.scratch.ptr + sh.starts_bytes);
  p.part_o = (float *)((char *)p.cuts + sh.cuts_bytes);
  p.part_ml = p.part_o + (size_t)2 * sh.ranges * a.g.n_kv_heads * sh.nw * 32 * a.head_dim;
  if (a.dtype == FOCUS_F32)
    a.head_dim == 64 ? run<float, 64>(s, a, p) : run<float, 128>(s, a, p);
  else
    a.head_dim == 64 ? run<bf16_t, 64>(s, a, p) : run<bf16_t, 128>(s, a, p);
}

}  // namespace fk
