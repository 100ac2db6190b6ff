// Products with microscaled 4-bit (MXFP4) weights on the matrix cores: dense, and grouped by expert.
//
// Two forms.  bf16 rows: codes become bf16 in registers (a 4-bit float times a power of two is exact in bf16) and go through
// v_mfma_f32_32x32x16_bf16.  MXFP4 rows: codes and scales go as they are through v_mfma_scale_f32_32x32x64_f8f6f4, four times the rate.
#include <algorithm>
#include <type_traits>

#include "focus_mx.h"

namespace fk {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

#define FK_LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))
constexpr int vmcnt_imm(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }   // s_waitcnt vmcnt(n) only
constexpr unsigned kOutside = 0x80000000u;   // an offset beyond every descriptor: the load returns zeros

// ---------------------------------------------------------------------------------------------
// bf16 rows x MXFP4 weights.
struct RowsArgs {
  const bf16_t *A;
  int64_t lda;
  const int32_t *src;                 // grouped: sorted row -> row of A, or null (rows in place)
  unsigned a_bytes;                   // with src: size of A
  const unsigned char *codes, *scales;
  int N, K;                           // of one expert's matrix
  Rows rows;                          // dense
  const int32_t *offs, *count, *tile_e, *tile_m0, *n_tiles;   // grouped
  int tiles_m, tiles_n, splits;
  void *out;
  int64_t ldo;
  size_t split_stride;                // fp32 partial sums of split s at out + s * split_stride
};
enum { RM_STORE, RM_STORE_F32, RM_ADD_F32, RM_SILU, RM_PARTIAL };

// the 8 scales of blocks b0 .. b0 + 7 of a row of `blocks`; those beyond the row are 0 (2^-127: their codes are zeros)
__device__ __forceinline__ uint64_t eight_scales(const unsigned char *row, int b0, int blocks) {
  uint64_t v = 0;
  if (blocks >= 8) {
    const int over = max(0, b0 + 8 - blocks);
    __builtin_memcpy(&v, row + (b0 - over), 8);
    return over >= 8 ? 0 : v >> (8 * over);
  }
  for (int j = 0; j < 8; ++j)
    if (b0 + j < blocks) v |= (uint64_t)row[b0 + j] << (8 * j);
  return v;
}

// A workgroup (4 wavefronts) takes up to BM rows and 128 CT rows of W; the wavefronts lie side by side, each BM x 32 CT, so that every code is
// read and converted by one wavefront; tile rows of 32 that hold no rows are skipped.  K goes in steps of 64 (128 bytes of a row of A, through LDS,
// DA steps ahead) and slabs of 256 (128 bytes of a row of W: a whole line, straight into registers, a slab ahead).  Lane l multiplies elements
// 32 h .. 32 h + 31 of a step, h = l / 32: one block of its weight row, so one scale; the order of the elements within a step is the same for
// both operands and does not matter otherwise.
constexpr int kAhead = 4;      // steps between asking for rows and using them: those of a slab

template <int BM, int CT, int MODE, bool GROUPED, bool WHOLE>      // WHOLE: K is a multiple of 256
__global__ __launch_bounds__(256, 2) void k_mx_rows(RowsArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)   // buffer-resource builtins exist in the device pass only
  constexpr int TM = BM / 32, DA = kAhead, SA = DA + 1, ASTAGE = BM * 128;
  constexpr bool SILU = MODE == RM_SILU;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[SA * ASTAGE];
  const int splits = GROUPED ? 1 : g.splits;
  const int M = GROUPED ? 0 : g.rows.count ? min(*g.rows.count, g.rows.cap) : g.rows.cap;
  const int tiles_m = GROUPED ? *g.n_tiles : (M + BM - 1) / BM, total = tiles_m * g.tiles_n * splits, per_xcd = (total + 7) / 8;
  // XCD x (workgroups x, x + 8, ...) takes a contiguous range of the work: workgroups that read the same rows share an L2
  const int item = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if ((int)(blockIdx.x / 8) >= per_xcd || item >= total) return;
  const int split = item % splits, t = item / splits / g.tiles_n, nt = item / splits % g.tiles_n;
  int e = 0, row0 = t * BM, valid;
  if (GROUPED) {
    e = g.tile_e[t];
    const int m0 = g.tile_m0[t];
    row0 = g.offs[e] + m0;
    valid = min(BM, g.count[e] - m0);
  } else {
    valid = min(BM, M - row0);
  }
  const int N = g.N, K = g.K, n0 = nt * (SILU ? 64 * CT : 128 * CT), blocks = K / 32;
  const int slabs = (blocks + 7) / 8, per_split = (slabs + splits - 1) / splits, slab0 = split * per_split;
  const int my_slabs = min(slabs - slab0, per_split);                                // slabs of this workgroup (0 or less: zeros)
  const int my_steps = (min(K, (slab0 + my_slabs) * 256) - slab0 * 256 + 63) / 64;   // steps that hold anything
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int frow = lane & 31, h = lane >> 5, live = (valid + 31) / 32;
  const unsigned char *const codes = g.codes + (size_t)e * N * (size_t)(K / 2), *const scales = g.scales + (size_t)e * N * (size_t)blocks;
  const bool gather = GROUPED && g.src;
  const bf16_t *const A = gather ? g.A : g.A + (size_t)row0 * g.lda;
  __amdgpu_buffer_rsrc_t rs_a = __builtin_amdgcn_make_buffer_rsrc((void *)A, 0, gather ? g.a_bytes : (unsigned)(((int64_t)(valid - 1) * g.lda + K) * 2), 0x00020000);
  __amdgpu_buffer_rsrc_t rs_w = __builtin_amdgcn_make_buffer_rsrc((void *)codes, 0, (unsigned)N * (unsigned)(K / 2), 0x00020000);
  __amdgpu_buffer_rsrc_t rs_s = __builtin_amdgcn_make_buffer_rsrc((void *)scales, 0, (unsigned)N * (unsigned)blocks, 0x00020000);
  // chunk (8 elements) of a step that this lane fetches for row 32 q + 8 wave + lane / 8 of the tile: swizzled so that LDS reads spread over
  // the banks (16 q + 4 wave + lane / 16 is half the row)
  const int ca = (lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7);
  unsigned voa[TM];
#pragma unroll
  for (int q = 0; q < TM; ++q) {
    const int r = q * 32 + wave * 8 + (lane >> 3), srow = r < valid ? (gather ? g.src[row0 + r] : r) : -1;
    voa[q] = srow < 0 ? kOutside : (unsigned)srow * (unsigned)g.lda * 2u + ca * 16;
  }
  // the matrix row of this lane's column in column tile j.  SiLU*up: with two tiles a wavefront gate and up of the same 32 columns; with
  // one 16 gate rows, then the 16 matching up rows
  unsigned vow[CT], vos[CT];
#pragma unroll
  for (int j = 0; j < CT; ++j) {
    int row;
    if (SILU) {
      const int c = CT == 2 ? n0 + wave * 32 + frow : n0 + wave * 16 + (frow & 15);
      row = c < N / 2 ? (CT == 2 ? j : frow >> 4) * (N / 2) + c : -1;
    } else {
      const int c = n0 + (wave * CT + j) * 32 + frow;
      row = c < N ? c : -1;
    }
    vow[j] = row < 0 ? kOutside : (unsigned)row * (unsigned)(K / 2) + h * 16;
    vos[j] = (unsigned)max(row, 0) * (unsigned)blocks;
  }

  u32x4 w[CT][4];
  uint64_t sc[CT];
  // two chunks of a slab's codes, q and q + 1
  auto load_w = [&](int slab, int q0) __attribute__((always_inline)) {
    const unsigned so = slab < my_slabs ? (unsigned)(slab0 + slab) * 128u : kOutside;
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int q = q0; q < q0 + 2; ++q)
        w[j][q] = __builtin_amdgcn_raw_buffer_load_b128(rs_w, !WHOLE && (slab0 + slab) * 8 + 2 * q + h >= blocks ? kOutside : vow[j] + q * 32, so, 0);
  };
  auto load_scales = [&](int slab) __attribute__((always_inline)) {
    const int b0 = (slab0 + min(slab, my_slabs - 1)) * 8;
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      if (WHOLE) sc[j] = __builtin_bit_cast(uint64_t, __builtin_amdgcn_raw_buffer_load_b64(rs_s, vos[j], b0, 0));
      else sc[j] = eight_scales(scales + vos[j], b0, blocks);
    }
  };

  f32x16 acc[TM][CT];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  const int swz_a = (frow >> 1) & 7;
  // L: tile rows of 32 that hold rows.  The loop exists once for each, since a branch around each tile row kept the fragments' LDS reads
  // from being asked for ahead.
  auto multiply = [&](auto rows_live) __attribute__((always_inline)) {
    constexpr int L = decltype(rows_live)::value;
    auto issue_a = [&](int step, int stage) __attribute__((always_inline)) {
      const int k0 = slab0 * 256 + step * 64;
      const unsigned so = step < my_steps ? (unsigned)k0 * 2u : kOutside;
      const bool half = !WHOLE && k0 + 32 >= K;           // the second block of the step does not exist
#pragma unroll
      for (int q = 0; q < L; ++q)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_a, FK_LDS_PTR(lds + stage * ASTAGE + (q * 4 + wave) * 1024), 16, half && ca >= 4 ? kOutside : voa[q], so, 0, 0);
    };
    // in the order in which the loop asks for them, so that its count of younger loads holds from the first step on
#pragma unroll
    for (int s = 0; s < DA; ++s) {
      issue_a(s, s);
      if (s & 1) load_w(0, s - 1);
      if (s == 3) load_scales(0);
    }
    int sa = 0, la = DA % SA;       // stages of this step's rows and of the loads it makes
    for (int slab = 0; slab < my_slabs; ++slab) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        // younger than the rows of this step: those of the three steps after it, four chunks of codes and a slab's scales
        __builtin_amdgcn_s_waitcnt(vmcnt_imm((DA - 1) * L + (WHOLE ? 5 : 4) * CT));
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // everyone has finished the step before
        issue_a(4 * slab + q + DA, la);
        const unsigned char *pa = lds + sa * ASTAGE;
        if (WHOLE || 4 * slab + q < my_steps) {
          float scale[CT];
#pragma unroll
          for (int j = 0; j < CT; ++j) {
            const unsigned x = (unsigned)((sc[j] >> (8 * h)) >> (32 * (q >> 1)));       // byte 2 (q & 1) is the scale of block 2 q + h
            scale[j] = __uint_as_float(((q & 1) ? x << 7 : x << 23) & 0x7F800000u);
          }
#pragma unroll
          for (int ks = 0; ks < 4; ++ks) {
            bf16x8 fb[CT], fa[L];
#pragma unroll
            for (int i = 0; i < L; ++i) fa[i] = *(const bf16x8 *)(pa + (i * 32 + frow) * 128 + (((4 * h + ks) ^ swz_a) << 4));
#pragma unroll
            for (int j = 0; j < CT; ++j) {
              const unsigned c = w[j][q][ks];
              const bf16x2 b0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale[j], 0), b1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale[j], 1);
              const bf16x2 b2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale[j], 2), b3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale[j], 3);
              fb[j] = bf16x8{b0[0], b0[1], b1[0], b1[1], b2[0], b2[1], b3[0], b3[1]};
            }
#pragma unroll
            for (int i = 0; i < L; ++i)
#pragma unroll
              for (int j = 0; j < CT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[i], fb[j], acc[i][j], 0, 0, 0);
          }
        }
        // into the registers just used
        if (q & 1) load_w(slab + 1, q - 1);
        if (q == 3) load_scales(slab + 1);
        sa = sa == SA - 1 ? 0 : sa + 1;
        la = la == SA - 1 ? 0 : la + 1;
      }
    }
  };
  if (my_slabs <= 0) {}
  else if (TM == 1 || live == 1) multiply(std::integral_constant<int, 1>());
  else if (live == 2) multiply(std::integral_constant<int, TM < 2 ? 1 : 2>());
  else if (live == 3) multiply(std::integral_constant<int, TM < 3 ? 1 : 3>());
  else multiply(std::integral_constant<int, TM>());
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  // register r of lane l is C[8 (r / 4) + 4 (l / 32) + r % 4][l % 32] of its 32 x 32 tile
  if (SILU) {
    // one column tile: lanes 0..15 of a half hold gate columns, 16..31 the matching up columns; exchanging halves between two registers gives
    // the lower lanes both numbers of register r and the upper lanes both of register r + 1
    const int gn = CT == 2 ? n0 + wave * 32 + frow : n0 + wave * 16 + (lane & 15);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += CT == 2 ? 1 : 2) {
        float ga = acc[i][0][r], up = acc[i][CT - 1][r];
        int rr = r;
        if (CT == 1) {
          const u32x2 x = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][0][r]), __float_as_uint(acc[i][0][(r + 1) & 15]), false, false);
          ga = __uint_as_float(x[0]); up = __uint_as_float(x[1]);
          rr = r + ((lane >> 4) & 1);
        }
        const int gm = i * 32 + 8 * (rr >> 2) + 4 * h + (rr & 3);
        // exp overflows to infinity and the quotient to 0 for a large negative gate
        if (gm < valid && gn < N / 2) ((bf16_t *)g.out)[(size_t)(row0 + gm) * g.ldo + gn] = (bf16_t)(ga / (1.0f + __expf(-ga)) * up);
      }
    return;
  }
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j) {
      const int gn = n0 + (wave * CT + j) * 32 + frow;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int gm = i * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
        if (gm < valid && gn < N) {
          const size_t at = (size_t)(row0 + gm) * g.ldo + gn;
          if (MODE == RM_STORE) ((bf16_t *)g.out)[at] = (bf16_t)acc[i][j][r];
          else if (MODE == RM_ADD_F32) ((float *)g.out)[at] += acc[i][j][r];
          else (MODE == RM_PARTIAL ? (float *)g.out + (size_t)split * g.split_stride : (float *)g.out)[at] = acc[i][j][r];
        }
      }
    }
#endif
}

template <int BM, int CT, int MODE, bool GROUPED>
void launch_rows(hipStream_t s, RowsArgs g, int tile_slots) {
  g.tiles_n = MODE == RM_SILU ? (g.N / 2 + 64 * CT - 1) / (64 * CT) : (g.N + 128 * CT - 1) / (128 * CT);
  const int grid = (tile_slots * g.tiles_n * (GROUPED ? 1 : g.splits) + 7) / 8 * 8;
  if (g.K % 256 == 0) k_mx_rows<BM, CT, MODE, GROUPED, true><<<grid, 256, 0, s>>>(g);
  else k_mx_rows<BM, CT, MODE, GROUPED, false><<<grid, 256, 0, s>>>(g);
}
template <int BM, int CT>
void launch_rows(hipStream_t s, int mode, const RowsArgs &g, int tile_slots) {
  if (mode == RM_STORE) launch_rows<BM, CT, RM_STORE, false>(s, g, tile_slots);
  else if (mode == RM_STORE_F32) launch_rows<BM, CT, RM_STORE_F32, false>(s, g, tile_slots);
  else if (mode == RM_ADD_F32) launch_rows<BM, CT, RM_ADD_F32, false>(s, g, tile_slots);
  else if (mode == RM_SILU) launch_rows<BM, CT, RM_SILU, false>(s, g, tile_slots);
  else launch_rows<BM, CT, RM_PARTIAL, false>(s, g, tile_slots);
}

// ---------------------------------------------------------------------------------------------
// MXFP4 rows x MXFP4 weights: 2 x 2 wavefronts, slabs of 256 elements (128 bytes a row).  Lane l supplies row l % 32 and block 2 j + l / 32 of the j-th
// quarter of a slab: 16 bytes of codes and one scale.
struct MxArgs {
  const unsigned char *A, *a_scales, *W, *w_scales;
  int M, N, K;
  int tiles_m, tiles_n, splits;
  void *out;
  int64_t ldo;
  size_t split_stride;
};
enum { XM_STORE, XM_STORE_F32, XM_PARTIAL };

template <int BM, int BN, int MODE>
__global__ __launch_bounds__(256, BM == 256 ? 1 : 2) void k_mx_mx(MxArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32, IA = BM / 32, IB = BN / 32;
  constexpr int ASTAGE = BM * 128, WSTAGE = BN * 128, WBASE = 2 * ASTAGE;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * (BM + BN) * 128];
  const int splits = g.splits, tiles_n = g.tiles_n, total = g.tiles_m * tiles_n * splits, per_xcd = (total + 7) / 8;
  const int item = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if ((int)(blockIdx.x / 8) >= per_xcd || item >= total) return;
  // tiles in groups of 8 tile rows, so that the panels of an XCD's range stay in its L2
  constexpr int GROUP = 8;
  const int split = item % splits, tile = item / splits;
  const int in_group = tile % (GROUP * tiles_n), first_m = tile / (GROUP * tiles_n) * GROUP, gsz = min(g.tiles_m - first_m, GROUP);
  const int m0 = (first_m + in_group % gsz) * BM, n0 = in_group / gsz * BN;
  const int M = g.M, N = g.N, K = g.K, blocks = K / 32, valid_m = min(BM, M - m0), valid_n = min(BN, N - n0);
  const int slabs = (blocks + 7) / 8, per_split = (slabs + splits - 1) / splits, slab0 = split * per_split, mine = min(slabs - slab0, per_split);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (wave >> 1) * WM, wn = (wave & 1) * WN, frow = lane & 31, h = lane >> 5;
  const unsigned char *const A = g.A + (size_t)m0 * (K / 2), *const W = g.W + (size_t)n0 * (K / 2);
  __amdgpu_buffer_rsrc_t rs_a = __builtin_amdgcn_make_buffer_rsrc((void *)A, 0, (unsigned)valid_m * (unsigned)(K / 2), 0x00020000);
  __amdgpu_buffer_rsrc_t rs_w = __builtin_amdgcn_make_buffer_rsrc((void *)W, 0, (unsigned)valid_n * (unsigned)(K / 2), 0x00020000);
  // chunk = block of 32 elements; rows beyond the matrix lie outside the descriptors
  const int chunk = (lane & 7) ^ ((lane >> 4) & 3);       // r = 8 q' + lane / 8: (r >> 1) & 7 = 4 (q' & 1) + (lane >> 4)
  auto issue = [&](int slab, int stage) {
    const unsigned so = slab < mine ? (unsigned)(slab0 + slab) * 128u : kOutside;
    const int left = blocks - (slab0 + slab) * 8;          // blocks of this slab that exist
#pragma unroll
    for (int q = 0; q < IA; ++q) {
      const int r = (wave * IA + q) * 8 + (lane >> 3), c = chunk ^ (4 * ((wave * IA + q) & 1));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_a, FK_LDS_PTR(lds + stage * ASTAGE + (wave * IA + q) * 1024), 16, c < left ? (unsigned)r * (unsigned)(K / 2) + c * 16 : kOutside, so, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < IB; ++q) {
      const int r = (wave * IB + q) * 8 + (lane >> 3), c = chunk ^ (4 * ((wave * IB + q) & 1));
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_w, FK_LDS_PTR(lds + WBASE + stage * WSTAGE + (wave * IB + q) * 1024), 16, c < left ? (unsigned)r * (unsigned)(K / 2) + c * 16 : kOutside, so, 0, 0);
    }
  };
  const unsigned char *sa[TM], *sb[TN];
#pragma unroll
  for (int i = 0; i < TM; ++i) sa[i] = g.a_scales + (size_t)(m0 + min(wm + i * 32 + frow, valid_m - 1)) * blocks;
#pragma unroll
  for (int j = 0; j < TN; ++j) sb[j] = g.w_scales + (size_t)(n0 + min(wn + j * 32 + frow, valid_n - 1)) * blocks;
  uint64_t ca[TM], cb[TN];
  auto scales = [&](int slab) {
    const int b0 = (slab0 + min(slab, mine - 1)) * 8;
#pragma unroll
    for (int i = 0; i < TM; ++i) ca[i] = eight_scales(sa[i], b0, blocks);
#pragma unroll
    for (int j = 0; j < TN; ++j) cb[j] = eight_scales(sb[j], b0, blocks);
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const int swz = (frow >> 1) & 7;
  if (mine > 0) {
    issue(0, 0);
    scales(0);
  }
  for (int slab = 0; slab < mine; ++slab) {
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    uint64_t na[TM], nb[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) na[i] = ca[i] >> (8 * h);       // byte 2 j of the shifted scales belongs to this lane's half
#pragma unroll
    for (int j = 0; j < TN; ++j) nb[j] = cb[j] >> (8 * h);
    issue(slab + 1, (slab + 1) & 1);
    scales(slab + 1);
    const unsigned char *pa = lds + (slab & 1) * ASTAGE, *pw = lds + WBASE + (slab & 1) * WSTAGE;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      i32x8 fa[TM], fb[TN];
      const int ch = ((2 * ks + h) ^ swz) << 4;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const u32x4 v = *(const u32x4 *)(pa + (wm + i * 32 + frow) * 128 + ch);
        fa[i] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
      }
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const u32x4 v = *(const u32x4 *)(pw + (wn + j * 32 + frow) * 128 + ch);
        fb[j] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
          const int xa = (int)(na[i] >> (32 * (ks >> 1))), xb = (int)(nb[j] >> (32 * (ks >> 1)));
          if (ks & 1) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa[i], fb[j], acc[i][j], 4, 4, 2, xa, 2, xb);
          else acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fa[i], fb[j], acc[i][j], 4, 4, 0, xa, 0, xb);
        }
    }
  }
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int gn = wn + j * 32 + frow;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int gm = wm + i * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
        if (gm < valid_m && gn < valid_n) {
          const size_t at = (size_t)(m0 + gm) * g.ldo + n0 + gn;
          if (MODE == XM_STORE) ((bf16_t *)g.out)[at] = (bf16_t)acc[i][j][r];
          else (MODE == XM_PARTIAL ? (float *)g.out + (size_t)split * g.split_stride : (float *)g.out)[at] = acc[i][j][r];
        }
      }
    }
#endif
}

template <int BM, int BN>
void launch_mx(hipStream_t s, int mode, MxArgs g) {
  g.tiles_m = (g.M + BM - 1) / BM;
  g.tiles_n = (g.N + BN - 1) / BN;
  const int grid = (g.tiles_m * g.tiles_n * g.splits + 7) / 8 * 8;
  if (mode == XM_STORE) k_mx_mx<BM, BN, XM_STORE><<<grid, 256, 0, s>>>(g);
  else if (mode == XM_STORE_F32) k_mx_mx<BM, BN, XM_STORE_F32><<<grid, 256, 0, s>>>(g);
  else k_mx_mx<BM, BN, XM_PARTIAL><<<grid, 256, 0, s>>>(g);
}

// ---------------------------------------------------------------------------------------------
// Adds the parts of a cut K in part order and does the epilogue.
template <int EPI>
__global__ __launch_bounds__(256) void k_mx_reduce(const float *__restrict__ part, int splits, size_t stride, Rows rows, int n, void *out, int64_t ldo) {
  const int M = rows.count ? min(*rows.count, rows.cap) : rows.cap, cols = EPI == MX_SILU_MUL ? n / 2 : n;
  const int64_t total = (int64_t)M * cols;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / cols, col = i - row * cols;
    const float *p = part + row * n + col;
    float v = 0.f, u = 0.f;
    for (int k = 0; k < splits; ++k) {
      v += p[(size_t)k * stride];
      if (EPI == MX_SILU_MUL) u += p[(size_t)k * stride + n / 2];
    }
    const size_t at = (size_t)row * ldo + col;
    if (EPI == MX_STORE) ((bf16_t *)out)[at] = (bf16_t)v;
    else if (EPI == MX_STORE_F32) ((float *)out)[at] = v;
    else if (EPI == MX_ADD_F32) ((float *)out)[at] += v;
    else ((bf16_t *)out)[at] = (bf16_t)(v / (1.0f + __expf(-v)) * u);
  }
}

void launch_reduce(hipStream_t s, int epi, const float *part, int splits, size_t stride, Rows rows, int n, void *out, int64_t ldo) {
  const int64_t total = (int64_t)rows.cap * (epi == MX_SILU_MUL ? n / 2 : n);
  const int grid = (int)std::min<int64_t>((total + 255) / 256, 4096);
  if (epi == MX_STORE) k_mx_reduce<MX_STORE><<<grid, 256, 0, s>>>(part, splits, stride, rows, n, out, ldo);
  else if (epi == MX_STORE_F32) k_mx_reduce<MX_STORE_F32><<<grid, 256, 0, s>>>(part, splits, stride, rows, n, out, ldo);
  else if (epi == MX_ADD_F32) k_mx_reduce<MX_ADD_F32><<<grid, 256, 0, s>>>(part, splits, stride, rows, n, out, ldo);
  else k_mx_reduce<MX_SILU_MUL><<<grid, 256, 0, s>>>(part, splits, stride, rows, n, out, ldo);
}

// Parts of K for `tiles` workgroups of which `resident` run at once: as many as fill the chip, each with 2 slabs at least.
int parts_of(int tiles, int resident, int slabs) { return std::max(1, std::min(resident / std::max(1, tiles), slabs / 2)); }
// parts with no slab left over are dropped
int whole_parts(int parts, int slabs) { const int per = (slabs + parts - 1) / parts; return (slabs + per - 1) / per; }

struct Shape { int bm, bn, splits; };
Shape shape_of(int rows, int n, int k, bool a_mx) {
  if (a_mx) {
    const int t256 = ((rows + 255) / 256) * ((n + 255) / 256), slabs = (k / 32 + 7) / 8;
    if (t256 >= 192) return {256, 256, 1};
    const int tiles = ((rows + 127) / 128) * ((n + 127) / 128);
    return {128, 128, whole_parts(parts_of(tiles, 512, slabs), std::max(1, slabs))};
  }
  const int bm = rows <= 32 ? 32 : 128, slabs = (k / 32 + 7) / 8, tiles_m = (rows + bm - 1) / bm, wide = tiles_m * ((n + 255) / 256);
  if (bm == 128 && wide >= 256) return {bm, 256, 1};
  return {bm, 128, whole_parts(parts_of(tiles_m * ((n + 127) / 128), 512, slabs), std::max(1, slabs))};
}

}  // namespace

size_t mx_gemm_scratch(int rows, int n, int k, bool a_mx) {
  const Shape p = shape_of(rows, n, k, a_mx);
  return p.splits > 1 ? (size_t)p.splits * rows * n * 4 : 0;
}

void mx_gemm(hipStream_t s, const void *a, const void *a_scales, int64_t lda, focus_mx w, int n, int k, Rows rows, int epilogue, void *out, int64_t ldo, Scratch scratch) {
  if (rows.cap <= 0 || n <= 0) return;
  const bool a_mx = a_scales != nullptr;
  Shape p = shape_of(rows.cap, n, k, a_mx);
  const size_t stride = (size_t)rows.cap * n;
  const int slabs = (k / 32 + 7) / 8;
  if (p.splits > 1) p.splits = whole_parts((int)std::max<size_t>(1, std::min<size_t>(p.splits, scratch.ptr ? scratch.bytes / (stride * 4) : 0)), slabs);
  const bool parts = p.splits > 1;
  if (a_mx) {
    MxArgs g{(const unsigned char *)a, (const unsigned char *)a_scales, (const unsigned char *)w.codes, (const unsigned char *)w.scales, rows.cap, n, k, 0, 0, p.splits,
             parts ? scratch.ptr : out, parts ? n : ldo, stride};
    const int mode = parts ? XM_PARTIAL : epilogue == MX_STORE ? XM_STORE : XM_STORE_F32;
    if (p.bm == 256) launch_mx<256, 256>(s, mode, g);
    else launch_mx<128, 128>(s, mode, g);
  } else {
    RowsArgs g{};
    g.A = (const bf16_t *)a; g.lda = lda; g.codes = (const unsigned char *)w.codes; g.scales = (const unsigned char *)w.scales; g.N = n; g.K = k; g.rows = rows;
    g.splits = p.splits; g.split_stride = stride; g.out = parts ? scratch.ptr : out; g.ldo = parts ? n : ldo;
    const int mode = parts ? RM_PARTIAL : epilogue == MX_STORE ? RM_STORE : epilogue == MX_STORE_F32 ? RM_STORE_F32 : epilogue == MX_ADD_F32 ? RM_ADD_F32 : RM_SILU;
    if (p.bm == 32) launch_rows<32, 1>(s, mode, g, (rows.cap + 31) / 32);
    else if (p.bn == 256) launch_rows<128, 2>(s, mode, g, (rows.cap + 127) / 128);
    else launch_rows<128, 1>(s, mode, g, (rows.cap + 127) / 128);
  }
  if (parts) launch_reduce(s, epilogue, (const float *)scratch.ptr, p.splits, stride, rows, n, out, ldo);
}

void mx_grouped(hipStream_t s, const MxGroups &g, const void *x, int64_t ldx, int n_rows, focus_mx gate_up, focus_mx down, int hidden, int ffn, void *act, float *y) {
  RowsArgs a{};
  a.A = (const bf16_t *)x; a.lda = ldx; a.src = g.src; a.a_bytes = (unsigned)(((int64_t)(n_rows - 1) * ldx + hidden) * 2);
  a.codes = (const unsigned char *)gate_up.codes; a.scales = (const unsigned char *)gate_up.scales;
  a.N = 2 * ffn; a.K = hidden; a.offs = g.offs; a.count = g.count; a.tile_e = g.tile_e; a.tile_m0 = g.tile_m0; a.n_tiles = g.n_tiles;
  a.splits = 1; a.out = act; a.ldo = ffn;
  launch_rows<128, 2, RM_SILU, true>(s, a, g.n_tile_slots);
  a.A = (const bf16_t *)act; a.lda = ffn; a.src = nullptr; a.a_bytes = 0;
  a.codes = (const unsigned char *)down.codes; a.scales = (const unsigned char *)down.scales;
  a.N = hidden; a.K = ffn; a.out = y; a.ldo = hidden;
  launch_rows<128, 2, RM_STORE_F32, true>(s, a, g.n_tile_slots);
}

// ---------------------------------------------------------------------------------------------
// Entries sorted by expert.  A workgroup counts 1024 entries per expert; a second launch adds up the counts and places the entries.  Which of a
// workgroup's entries of one expert comes first is left to the order of its LDS atomics: a row's sums do not depend on its place in a tile.
namespace {
constexpr int kChunk = 1024;

__global__ __launch_bounds__(kChunk) void k_mx_count(MxExperts a) {
  extern __shared__ int cnt[];
  const int E = a.n_experts, tid = threadIdx.x, M = a.rows.count ? min(*a.rows.count, a.rows.cap) : a.rows.cap, n = M * a.k;
  for (int e = tid; e < E; e += kChunk) cnt[e] = 0;
  __syncthreads();
  const int i = blockIdx.x * kChunk + tid;
  if (i < n) {
    const int e = a.experts[i];
    if (e >= 0 && e < E) atomicAdd(&cnt[e], 1);
  }
  __syncthreads();
  for (int e = tid; e < E; e += kChunk) a.hist[(size_t)blockIdx.x * E + e] = cnt[e];
}

// all[e]: rows of expert e; mine[e]: of the chunks before this one.  Exclusive sums over the experts of rows and of tiles, in LDS.
__global__ __launch_bounds__(kChunk) void k_mx_place(MxExperts a, int chunks, int tile_slots) {
  extern __shared__ int lds_place[];
  const int E = a.n_experts, tid = threadIdx.x, M = a.rows.count ? min(*a.rows.count, a.rows.cap) : a.rows.cap, n = M * a.k;
  int *all = lds_place, *next = all + E, *rows_lt = next + E, *tiles_lt = rows_lt + E;
  for (int e = tid; e < E; e += kChunk) {
    int before = 0, sum = 0;
    for (int c = 0; c < chunks; ++c) {
      const int v = a.hist[(size_t)c * E + e];
      before += c < (int)blockIdx.x ? v : 0;
      sum += v;
    }
    all[e] = sum;
    next[e] = before;
  }
  __syncthreads();
  if (tid < 64) {                       // one wavefront scans, 64 experts at a time
    int rows = 0, tiles = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
      const int e = e0 + tid, c = e < E ? all[e] : 0, t = (c + kMxTileRows - 1) / kMxTileRows;
      int r = c, q = t;
      for (int d = 1; d < 64; d <<= 1) {
        const int ro = __shfl_up(r, d), qo = __shfl_up(q, d);
        if (tid >= d) { r += ro; q += qo; }
      }
      if (e < E) { rows_lt[e] = rows + r - c; tiles_lt[e] = tiles + q - t; }
      rows += __shfl(r, 63);
      tiles += __shfl(q, 63);
    }
    if (blockIdx.x == 0 && tid == 0) { a.offs[E] = rows; *a.n_tiles = min(tiles, tile_slots); }
  }
  __syncthreads();
  for (int e = tid; e < E; e += kChunk) next[e] += rows_lt[e];
  if (blockIdx.x == 0)
    for (int e = tid; e < E; e += kChunk) {
      a.offs[e] = rows_lt[e];
      a.count[e] = all[e];
      for (int m = 0; m * kMxTileRows < all[e] && tiles_lt[e] + m < tile_slots; ++m) { a.tile_e[tiles_lt[e] + m] = e; a.tile_m0[tiles_lt[e] + m] = m * kMxTileRows; }
    }
  __syncthreads();
  const int i = blockIdx.x * kChunk + tid;
  if (i < n) {
    const int e = a.experts[i];
    int p = -1;
    if (e >= 0 && e < E) {
      p = atomicAdd(&next[e], 1);
      a.arow[p] = i / a.k;
    }
    a.pos[i] = p;
  }
}

// out[row] (+)= sum_j weight_j y[pos_j], j ascending; a workgroup takes 1024 columns of a row
template <typename T, bool ADD>
__global__ __launch_bounds__(256) void k_mx_combine(MxExperts a) {
  const int row = blockIdx.x, k = a.k, H = a.hidden;
  if (a.rows.count && row >= *a.rows.count) return;
  const int c = (blockIdx.y * 256 + threadIdx.x) * 4;
  if (c >= H) return;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j = 0; j < k; ++j) {
    const int p = a.pos[(size_t)row * k + j];
    if (p < 0) continue;
    const float w = a.weights[(size_t)row * k + j];
    const float4 v = *(const float4 *)(a.y + (size_t)p * H + c);
    acc.x += w * v.x; acc.y += w * v.y; acc.z += w * v.z; acc.w += w * v.w;
  }
  T *o = (T *)a.out + (size_t)row * a.ldo + c;
  const float v[4] = {acc.x, acc.y, acc.z, acc.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = ADD ? (T)((float)o[i] + v[i]) : (T)v[i];
}

int tile_slots_of(int entries, int E) { return entries / kMxTileRows + std::min(entries, E); }
}  // namespace

// Lays the work buffers out from `base`; returns their size.
static size_t lay(MxExperts &a, char *base, int rows) {
  const size_t ent = (size_t)rows * a.k, E = a.n_experts, chunks = (ent + kChunk - 1) / kChunk, tiles = tile_slots_of((int)ent, a.n_experts);
  size_t at = 0;
  auto take = [&](size_t bytes) { char *p = base + at; at += (bytes + 255) & ~(size_t)255; return p; };
  a.hist = (int32_t *)take(chunks * E * 4);
  a.offs = (int32_t *)take((E + 1) * 4);
  a.count = (int32_t *)take(E * 4);
  a.tile_e = (int32_t *)take(tiles * 4);
  a.tile_m0 = (int32_t *)take(tiles * 4);
  a.n_tiles = (int32_t *)take(4);
  a.pos = (int32_t *)take(ent * 4);
  a.arow = (int32_t *)take(ent * 4);
  a.act = take(ent * a.ffn * 2);
  a.y = (float *)take(ent * a.hidden * 4);
  return at;
}
size_t mx_experts_bytes(int n_experts, int hidden, int ffn, int n_rows, int k) {
  MxExperts a{};
  a.n_experts = n_experts; a.hidden = hidden; a.ffn = ffn; a.k = k;
  return lay(a, nullptr, n_rows);
}
void lay_mx_experts(MxExperts &a, void *workspace) { lay(a, (char *)workspace, a.rows.cap); }

void mx_experts(hipStream_t s, const MxExperts &a) {
  if (a.rows.cap <= 0) return;
  const int ent = a.rows.cap * a.k, chunks = (ent + kChunk - 1) / kChunk, slots = tile_slots_of(ent, a.n_experts);
  k_mx_count<<<chunks, kChunk, a.n_experts * 4, s>>>(a);
  k_mx_place<<<chunks, kChunk, a.n_experts * 16, s>>>(a, chunks, slots);
  mx_grouped(s, MxGroups{a.offs, a.count, a.tile_e, a.tile_m0, a.n_tiles, slots, a.arow}, a.x, a.ldx, a.rows.cap, a.gate_up, a.down, a.hidden, a.ffn, a.act, a.y);
  const dim3 grid(a.rows.cap, (a.hidden + 1023) / 1024);
  if (a.out_type == FOCUS_BF16) k_mx_combine<bf16_t, false><<<grid, 256, 0, s>>>(a);
  else if (a.add) k_mx_combine<float, true><<<grid, 256, 0, s>>>(a);
  else k_mx_combine<float, false><<<grid, 256, 0, s>>>(a);
}

}  // namespace fk
