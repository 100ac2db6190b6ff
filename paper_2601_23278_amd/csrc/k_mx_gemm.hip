// Products with microscaled 4-bit (MXFP4) weights on the matrix cores: dense, and grouped by expert.
//
// Two forms.  bf16 rows: codes become bf16 in registers (a 4-bit float times a power of two is exact in bf16) and go through
// v_mfma_f32_32x32x16_bf16.  MXFP4 rows: codes and scales go as they are through v_mfma_scale_f32_32x32x64_f8f6f4, four times the rate.
#include <algorithm>

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

// A workgroup (4 wavefronts) takes up to BM rows and 128 rows of W; the wavefronts lie side by side, each BM x 32, so that every code is
// converted once, and tile rows of 32 that hold no rows are skipped.  K goes in steps of 64 of the rows (128 bytes a row) and slabs of 128 of the
// codes (64 bytes a row), straight into LDS.  Lane l multiplies elements 32 h .. 32 h + 31 of a step, h = l / 32: one block of its weight
// row, so one scale; the order of the elements within a step is the same for both operands and does not matter otherwise.
constexpr int ahead_of(int bm) { return bm > 32 ? 2 : 6; }      // steps between asking for data and using it (even)
constexpr int rows_lds(int bm) { return (ahead_of(bm) + 1) * bm * 128 + (ahead_of(bm) / 2 + 2) * (8192 + 1024); }

template <int BM, int MODE, bool GROUPED, bool WHOLE>      // WHOLE: K is a multiple of 128
__global__ __launch_bounds__(256, 2) void k_mx_rows(RowsArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)   // buffer-resource builtins exist in the device pass only
  constexpr int TM = BM / 32, IA = BM / 32, DA = ahead_of(BM), SA = DA + 1, DW = DA / 2 + 1, SW = DW + 1;
  constexpr int ASTAGE = BM * 128, WSTAGE = 8192, SSTAGE = 1024, WBASE = SA * ASTAGE, SBASE = WBASE + SW * WSTAGE;
  constexpr bool SILU = MODE == RM_SILU;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[rows_lds(BM)];
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
  const int N = g.N, K = g.K, n0 = nt * (SILU ? 64 : 128), blocks = K / 32;
  const int slabs = (blocks + 3) / 4, per_split = (slabs + splits - 1) / splits, slab0 = split * per_split;
  const int my_slabs = min(slabs - slab0, per_split), steps = 2 * my_slabs;          // slabs of this workgroup (0 or less: zeros)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int frow = lane & 31, h = lane >> 5, live = (valid + 31) / 32;
  const unsigned char *const codes = g.codes + (size_t)e * N * (size_t)(K / 2), *const scales = g.scales + (size_t)e * N * (size_t)blocks;
  const bool gather = GROUPED && g.src;
  const bf16_t *const A = gather ? g.A : g.A + (size_t)row0 * g.lda;
  __amdgpu_buffer_rsrc_t rs_a = __builtin_amdgcn_make_buffer_rsrc((void *)A, 0, gather ? g.a_bytes : (unsigned)(((int64_t)(valid - 1) * g.lda + K) * 2), 0x00020000);
  __amdgpu_buffer_rsrc_t rs_w = __builtin_amdgcn_make_buffer_rsrc((void *)codes, 0, (unsigned)N * (unsigned)(K / 2), 0x00020000);
  __amdgpu_buffer_rsrc_t rs_s = __builtin_amdgcn_make_buffer_rsrc((void *)scales, 0, (unsigned)N * (unsigned)blocks, 0x00020000);
  // chunk (8 elements) of a step that this lane fetches for row r of the tile: swizzled so that LDS reads spread over the banks
  unsigned voa[IA];
  int ca[IA];
#pragma unroll
  for (int q = 0; q < IA; ++q) {
    const int r = (wave * IA + q) * 8 + (lane >> 3);
    ca[q] = (lane & 7) ^ ((r >> 1) & 7);
    const int srow = r < valid ? (gather ? g.src[row0 + r] : r) : -1;
    voa[q] = srow < 0 ? kOutside : (unsigned)srow * (unsigned)g.lda * 2u + ca[q] * 16;
  }
  // the matrix row of row r (0..31) of this wavefront's columns: with SiLU*up 16 gate rows, then the 16 matching up rows
  auto weight_row = [&](int r) {
    if (SILU) {
      const int c = n0 + wave * 16 + (r & 15);
      return c < N / 2 ? (r >> 4) * (N / 2) + c : -1;
    }
    const int c = n0 + wave * 32 + r;
    return c < N ? c : -1;
  };
  unsigned vow[2];
  const int cw[2] = {(lane & 3) ^ ((lane >> 4) & 3), (lane & 3) ^ ((lane >> 4) & 3)};
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int wr = weight_row(p * 16 + (lane >> 2));
    vow[p] = wr < 0 ? kOutside : (unsigned)wr * (unsigned)(K / 2) + cw[p] * 16;
  }
  const int srow = weight_row(frow);
  const unsigned vos = srow < 0 || h ? kOutside : (unsigned)srow * (unsigned)blocks;

  auto issue_a = [&](int step, int stage) {
    const int k0 = slab0 * 128 + step * 64;
    const unsigned so = step < steps && k0 < K ? (unsigned)k0 * 2u : kOutside;
    const bool half = !WHOLE && k0 + 32 >= K;           // the second block of the step does not exist
#pragma unroll
    for (int q = 0; q < IA; ++q)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_a, FK_LDS_PTR(lds + stage * ASTAGE + (wave * IA + q) * 1024), 16, half && ca[q] >= 4 ? kOutside : voa[q], so, 0, 0);
  };
  auto issue_w = [&](int slab, int stage, int part) {
    const unsigned so = slab < my_slabs ? (unsigned)(slab0 + slab) * 64u : kOutside;
    const unsigned v = !WHOLE && (slab0 + slab) * 4 + cw[part] >= blocks ? kOutside : vow[part];
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_w, FK_LDS_PTR(lds + WBASE + stage * WSTAGE + (wave * 2 + part) * 1024), 16, v, so, 0, 0);
  };
  auto issue_s = [&](int slab, int stage) {
    unsigned char *to = lds + SBASE + stage * SSTAGE + wave * 256;
    if (WHOLE) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_s, FK_LDS_PTR(to), 4, vos, slab < my_slabs ? (unsigned)(slab0 + slab) * 4u : kOutside, 0, 0);
    } else if (slab < my_slabs && h == 0) {              // rows of scales are not aligned: byte by byte
      unsigned s = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int b = (slab0 + slab) * 4 + j;
        s |= (unsigned)__builtin_amdgcn_raw_buffer_load_b8(rs_s, b < blocks && vos != kOutside ? vos + b : kOutside, 0, 0) << (8 * j);
      }
      *(unsigned *)(to + frow * 4) = s;
    }
  };

  f32x16 acc[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;

  // step s asks for the rows of step s + DA and half of the codes of slab s / 2 + DW; even steps also for that slab's scales.  So a step's codes
  // and scales were asked for before its rows.
  issue_w(0, 0, 0);
  issue_w(0, 0, 1);
  issue_s(0, 0);
#pragma unroll
  for (int s = 0; s < DA; ++s) {
    issue_a(s, s);
    issue_w(s / 2 + 1, s / 2 + 1, s & 1);
    if (!(s & 1)) issue_s(s / 2 + 1, s / 2 + 1);
  }
  constexpr int FLY = WHOLE ? DA / 2 * (IA + 1) + (DA / 2 - 1) * (IA + 2) + 2 : DA / 2 * (IA + 1) + (DA / 2 - 1) * (IA + 1) + 1;
  int sa = 0, sw = 0, la = DA % SA, lw = DW % SW;       // stages of this step's data and of the loads it makes
  const int swz_a = (frow >> 1) & 7, swz_w = (frow >> 2) & 3;
  for (int slab = 0; slab < my_slabs; ++slab) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      // all but the youngest FLY loads have landed: the rows of this step, and older ones; everyone has finished the step before
      __builtin_amdgcn_s_waitcnt(vmcnt_imm(FLY));
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      issue_a(2 * slab + q + DA, la);
      issue_w(slab + DW, lw, q);
      if (q == 0) issue_s(slab + DW, lw);
      const unsigned char *pa = lds + sa * ASTAGE, *pw = lds + WBASE + sw * WSTAGE + (wave * 32 + frow) * 64;
      const unsigned sc = *(const unsigned *)(lds + SBASE + sw * SSTAGE + wave * 256 + frow * 4);
      const u32x4 wv = *(const u32x4 *)(pw + (((2 * q + h) ^ swz_w) << 4));
      const float scale = __uint_as_float(((sc >> (8 * (2 * q + h))) & 255u) << 23);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        const bf16x2 b0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wv[ks], scale, 0), b1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wv[ks], scale, 1);
        const bf16x2 b2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wv[ks], scale, 2), b3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(wv[ks], scale, 3);
        const bf16x8 fb = {b0[0], b0[1], b1[0], b1[1], b2[0], b2[1], b3[0], b3[1]};
#pragma unroll
        for (int i = 0; i < TM; ++i)
          if (i < live) {
            const bf16x8 fa = *(const bf16x8 *)(pa + (i * 32 + frow) * 128 + (((4 * h + ks) ^ swz_a) << 4));
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa, fb, acc[i], 0, 0, 0);
          }
      }
      sa = sa == SA - 1 ? 0 : sa + 1;
      la = la == SA - 1 ? 0 : la + 1;
    }
    sw = sw == SW - 1 ? 0 : sw + 1;
    lw = lw == SW - 1 ? 0 : lw + 1;
  }
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  // register r of lane l is C[8 (r / 4) + 4 (l / 32) + r % 4][l % 32] of its 32 x 32 tile
  if (SILU) {
    // lanes 0..15 of a half hold gate columns, 16..31 the matching up columns: exchanging halves between two registers gives the lower
    // lanes both numbers of register r and the upper lanes both of register r + 1
    const int gn = n0 + wave * 16 + (lane & 15);
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const u32x2 x = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[i][r]), __float_as_uint(acc[i][r + 1]), false, false);
        const float ga = __uint_as_float(x[0]), up = __uint_as_float(x[1]);
        const int rr = r + ((lane >> 4) & 1), gm = i * 32 + 8 * (rr >> 2) + 4 * h + (rr & 3);
        // exp overflows to infinity and the quotient to 0 for a large negative gate
        if (gm < valid && gn < N / 2) ((bf16_t *)g.out)[(size_t)(row0 + gm) * g.ldo + gn] = (bf16_t)(ga / (1.0f + __expf(-ga)) * up);
      }
    return;
  }
  const int gn = n0 + wave * 32 + frow;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int gm = i * 32 + 8 * (r >> 2) + 4 * h + (r & 3);
      if (gm < valid && gn < N) {
        const size_t at = (size_t)(row0 + gm) * g.ldo + gn;
        if (MODE == RM_STORE) ((bf16_t *)g.out)[at] = (bf16_t)acc[i][r];
        else if (MODE == RM_ADD_F32) ((float *)g.out)[at] += acc[i][r];
        else (MODE == RM_PARTIAL ? (float *)g.out + (size_t)split * g.split_stride : (float *)g.out)[at] = acc[i][r];
      }
    }
#endif
}

template <int BM, int MODE, bool GROUPED>
void launch_rows(hipStream_t s, const RowsArgs &g, int tile_slots) {
  const int grid = (tile_slots * g.tiles_n * (GROUPED ? 1 : g.splits) + 7) / 8 * 8;
  if (g.K % 128 == 0) k_mx_rows<BM, MODE, GROUPED, true><<<grid, 256, 0, s>>>(g);
  else k_mx_rows<BM, MODE, GROUPED, false><<<grid, 256, 0, s>>>(g);
}
template <int BM>
void launch_rows(hipStream_t s, int mode, const RowsArgs &g, int tile_slots) {
  if (mode == RM_STORE) launch_rows<BM, RM_STORE, false>(s, g, tile_slots);
  else if (mode == RM_STORE_F32) launch_rows<BM, RM_STORE_F32, false>(s, g, tile_slots);
  else if (mode == RM_ADD_F32) launch_rows<BM, RM_ADD_F32, false>(s, g, tile_slots);
  else if (mode == RM_SILU) launch_rows<BM, RM_SILU, false>(s, g, tile_slots);
  else launch_rows<BM, RM_PARTIAL, false>(s, g, tile_slots);
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

// Parts of K for `tiles` workgroups of which `resident` run at once: as many as fill the chip, each with 4 slabs at least.
int parts_of(int tiles, int resident, int slabs) { return std::max(1, std::min(resident / std::max(1, tiles), slabs / 4)); }
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
  const int bm = rows <= 32 ? 32 : 128, slabs = (k / 32 + 3) / 4, tiles = ((rows + bm - 1) / bm) * ((n + 127) / 128);
  return {bm, 128, whole_parts(parts_of(tiles, 512, slabs), std::max(1, slabs))};
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
  const int slabs = (k / 32 + (a_mx ? 7 : 3)) / (a_mx ? 8 : 4);
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
    const bool silu = epilogue == MX_SILU_MUL && !parts;
    g.tiles_n = silu ? (n / 2 + 63) / 64 : (n + 127) / 128;
    const int mode = parts ? RM_PARTIAL : epilogue == MX_STORE ? RM_STORE : epilogue == MX_STORE_F32 ? RM_STORE_F32 : epilogue == MX_ADD_F32 ? RM_ADD_F32 : RM_SILU;
    if (p.bm == 32) launch_rows<32>(s, mode, g, (rows.cap + 31) / 32);
    else launch_rows<128>(s, mode, g, (rows.cap + 127) / 128);
  }
  if (parts) launch_reduce(s, epilogue, (const float *)scratch.ptr, p.splits, stride, rows, n, out, ldo);
}

void mx_grouped(hipStream_t s, const MxGroups &g, const void *x, int64_t ldx, int n_rows, focus_mx gate_up, focus_mx down, int hidden, int ffn, void *act, float *y) {
  RowsArgs a{};
  a.A = (const bf16_t *)x; a.lda = ldx; a.src = g.src; a.a_bytes = (unsigned)(((int64_t)(n_rows - 1) * ldx + hidden) * 2);
  a.codes = (const unsigned char *)gate_up.codes; a.scales = (const unsigned char *)gate_up.scales;
  a.N = 2 * ffn; a.K = hidden; a.offs = g.offs; a.count = g.count; a.tile_e = g.tile_e; a.tile_m0 = g.tile_m0; a.n_tiles = g.n_tiles;
  a.tiles_n = (ffn + 63) / 64; a.splits = 1; a.out = act; a.ldo = ffn;
  launch_rows<128, RM_SILU, true>(s, a, g.n_tile_slots);
  a.A = (const bf16_t *)act; a.lda = ffn; a.src = nullptr; a.a_bytes = 0;
  a.codes = (const unsigned char *)down.codes; a.scales = (const unsigned char *)down.scales;
  a.N = hidden; a.K = ffn; a.tiles_n = (hidden + 127) / 128; a.out = y; a.ldo = hidden;
  launch_rows<128, RM_STORE_F32, true>(s, a, g.n_tile_slots);
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
