// Products with microscaled 4-bit (MXFP4) weights on the matrix cores: dense, and grouped by expert.
//
// Two forms.  bf16 rows: codes become bf16 in registers (a 4-bit float times a power of two from 2^-127 on is exact in bf16 below 2^128, infinite from
// there on) and go through v_mfma_f32_32x32x16_bf16, which takes numbers below the smallest normal one.  MXFP4 rows: codes and scales go as they are through v_mfma_scale_f32_32x32x64_f8f6f4, four times the rate.
#include <algorithm>
#include <iterator>
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

// fp32 products of the routed experts that the memory-side cache still holds when they are added up (mx_down)
constexpr int64_t kMxSliceBytes = 136ll << 20;
#define FK_LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))
constexpr int vmcnt_imm(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }   // s_waitcnt vmcnt(n) only
constexpr unsigned kOutside = 0x80000000u;   // an offset beyond every descriptor: the load returns zeros

// A wavefront's results of 32 rows and 8 G columns into C, through LDS of its own (32 tile_pitch() bytes): value(g) of lane l are C[l % 32][8 g + 4 (l / 32) + 0 .. 3]
// (four registers of the product of transposed operands), so four neighbours go into LDS at once, and whole pieces of rows come out, 16 bytes a lane.
// Stored straight from the registers, an element per lane and instruction, with an address and two comparisons for each, 2048 x 24576 x 4096 with both
// operands in MXFP4 took a fifth longer (125 us against 104, in turn on one card).
// rows, cols: of the tile that exist; wide: the rows of C are 16-byte aligned.
#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ void wave_lds_order() {      // the lanes' traffic runs in order, only the compiler has to keep it so
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
#endif
template <typename T> constexpr int tile_pitch(int groups) { return groups * 8 * (int)sizeof(T) + 16; }      // rows of 128 bytes and more lie four banks apart
typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename T, bool ADD, int G, typename V>
__device__ __forceinline__ void store_tile(unsigned char *mine, const V &value, T *out, int64_t ldo, int rows, int cols, bool wide) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int P = tile_pitch<T>(G), PER = 16 / sizeof(T), LANES = G * 8 / PER, ROWS = 64 / LANES;      // elements a lane, lanes a row, rows an instruction
  typedef T tx4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 63, frow = lane & 31, h = lane >> 5;
#pragma unroll
  for (int g = 0; g < G; ++g) *(tx4 *)(mine + frow * P + (8 * g + 4 * h) * (int)sizeof(T)) = __builtin_convertvector(value(g), tx4);
  wave_lds_order();
  const int row0 = lane / LANES, col = lane % LANES * PER;
  T *o = out + (int64_t)row0 * ldo + col;
#pragma unroll
  for (int it = 0; it < 32 / ROWS; ++it, o += ROWS * ldo) {
    typedef T txp __attribute__((ext_vector_type(PER)));
    txp v = *(const txp *)(mine + (it * ROWS + row0) * P + col * (int)sizeof(T));
    if (it * ROWS + row0 >= rows || col >= cols) continue;
    if (wide && col + PER <= cols) {
      if (ADD) v += *(const txp *)o;
      *(txp *)o = v;
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e)
        if (col + e < cols) o[e] = ADD ? (T)(o[e] + v[e]) : v[e];
    }
  }
  wave_lds_order();
#endif
}

// ---------------------------------------------------------------------------------------------
// bf16 rows x MXFP4 weights.
struct RowsArgs {
  const bf16_t *A;
  int64_t lda;
  const int32_t *src;                 // grouped: sorted row -> row of A, or null (rows in place)
  unsigned a_bytes;                   // with src: size of A
  const unsigned char *codes, *scales;
  int N, K;                           // of one expert's matrix
  int n_begin, n_end;                 // columns of C wanted; column n_begin is the first one written
  Rows rows;                          // dense
  const int2 *tiles;                  // grouped: first sorted row; expert and rows << 16
  const int32_t *n_tiles;
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
// read and converted by one wavefront; tile rows of 32 that hold no rows are skipped.  K goes in steps of 64 (128 bytes of a row of A) and slabs
// of four steps (128 bytes of a row of W), whole lines of both, straight into LDS: the rows three steps ahead, the codes kCodeStages slabs ahead of the
// registers that hold the slab in work.  (Codes read from memory into registers, a row per lane, cost the vector caches 64 lookups an instruction instead of
// 16: gate/up of 2048 rows through 8 of 256 experts each, 2048 -> 512, took 134 us instead of 105.)  Lane l multiplies elements 32 h .. 32 h + 31 of a step, h = l / 32: one
// block of its weight row, so one scale; the order of the elements within a step is the same for both operands and does not matter otherwise.
// Pipelined by hand: behind the MFMAs of 16 elements of K go the LDS reads of the rows' next fragments, the conversions of the next codes and the
// loads.  A step's last quarter begins with the only barrier: by then everyone has read all of the step's rows, whose stage is filled again right
// behind it, and the next step's rows have landed.  Codes are read and written by their own wavefront alone.
// What bounds it: few rows, the codes' way from memory (8 rows x 24576 x 4096, 54 MB: 15.0 us, 3.6 TB/s, two rounds of workgroups that each wait for
// their first slabs); many rows, the matrix units, busy in 67 % of the cycles (2048 x 24576 x 4096: 318 us, 1.30 PFLOP/s; a large bf16 library product 1.37); in
// between, both by halves (those gate/up rows, 69 GFLOP and 285 MB of codes: 96 us; the loads alone took 71 of 105, the arithmetic alone 75; the last round
// of workgroups leaves a fifth of the chip idle).
constexpr int kRowStages = 3;
constexpr int code_stages(int bm) { return bm > 32 ? 1 : 2; }
constexpr int rows_lds(int bm, int ct) { return kRowStages * bm * 128 + code_stages(bm) * ct * 16384; }

template <int BM, int CT, int MODE, bool GROUPED, bool WHOLE>      // WHOLE: K is a multiple of 256
__global__ __launch_bounds__(256, 2) void k_mx_rows(RowsArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)   // buffer-resource builtins exist in the device pass only
  constexpr int TM = BM / 32, SA = kRowStages, ASTAGE = BM * 128, SW = code_stages(BM), WSTAGE = CT * 4096, WBASE = SA * ASTAGE;
  constexpr bool SILU = MODE == RM_SILU;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[rows_lds(BM, CT)];
  const int splits = GROUPED ? 1 : g.splits;
  const int M = GROUPED ? 0 : g.rows.count ? min(*g.rows.count, g.rows.cap) : g.rows.cap;
  const int tile_at = blockIdx.x / 8 / g.tiles_n * 8 + blockIdx.x % 8;
  const int2 tile = GROUPED ? g.tiles[tile_at] : make_int2(0, 0);       // asked for together with the number of tiles: the list has room for every workgroup
  const int tiles_m = GROUPED ? *g.n_tiles : (M + BM - 1) / BM, total = tiles_m * g.tiles_n * splits, per_xcd = (total + 7) / 8;
  // XCD x has the workgroups x, x + 8, ...  Dense: it takes a contiguous range of the work, so that workgroups that read the same rows share an
  // L2.  Grouped: it takes the row tiles x, x + 8, ..., each with all its columns; the fullest tiles come first in the list, so that the
  // launch ends with short ones on every XCD.
  const int local = blockIdx.x / 8, item = (blockIdx.x % 8) * per_xcd + local;
  if (GROUPED ? tile_at >= tiles_m : local >= per_xcd || item >= total) return;
  const int split = item % splits, t = item / splits / g.tiles_n;
  const int nt = GROUPED ? local % g.tiles_n : item / splits % g.tiles_n;
  const int e = GROUPED ? tile.y & 0xFFFF : 0, row0 = GROUPED ? tile.x : t * BM, valid = GROUPED ? tile.y >> 16 : min(BM, M - row0);
  const int N = g.N, K = g.K, n0 = g.n_begin + nt * (SILU ? 64 * CT : 128 * CT), n_end = g.n_end, blocks = K / 32;
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
  // the matrix row of column r (0 .. 32 CT - 1) of this wavefront.  SiLU*up: with two column tiles gate and up of the same 32 columns; with one 16
  // gate rows, then the 16 matching up rows
  auto weight_row = [&](int r) __attribute__((always_inline)) {
    if (SILU) {
      const int c = CT == 2 ? n0 + wave * 32 + (r & 31) : n0 + wave * 16 + (r & 15);
      return c < n_end ? (CT == 2 ? r >> 5 : r >> 4) * (N / 2) + c : -1;
    }
    const int c = n0 + wave * 32 * CT + r;
    return c < n_end ? c : -1;
  };
  // chunk (block of 32) of a slab that this lane fetches for columns 8 q + lane / 8, q even and odd: swizzled like the rows' chunks
  const int cw = (lane & 7) ^ (lane >> 4);
  unsigned vow[4 * CT];
#pragma unroll
  for (int q = 0; q < 4 * CT; ++q) {
    const int row = weight_row(q * 8 + (lane >> 3));
    vow[q] = row < 0 ? kOutside : (unsigned)row * (unsigned)(K / 2) + (cw ^ (4 * (q & 1))) * 16;
  }
  // scales: with two column tiles the lower lanes fetch those of the first, the upper ones of the second
  const int srow = weight_row(CT == 2 ? lane : frow);
  const unsigned vos = (unsigned)max(srow, 0) * (unsigned)blocks;
  f32x16 acc[TM][CT];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < CT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  // L: tile rows of 32 that hold rows.  The loop exists once for each, since a branch around each tile row would part the pipeline.
  auto multiply = [&](auto rows_live) __attribute__((always_inline)) {
    constexpr int L = decltype(rows_live)::value, NMF = L * CT, PER = (3 + L) / L;      // PER: conversions behind an MFMA, four in L of them
    u32x4 w[CT][4];             // codes of the slab: chunk of each step
    u32x2 sc[CT];               // its scales, and those of the next slab as they were fetched
    u32x2 next_sc;
    u32x4 fb[2];                // CT = 2: of the two column tiles; CT = 1: of this quarter and the next
    // Fragments of this quarter and the next; with two column tiles and three or four tile rows a fragment's successor goes where it was, behind its
    // last MFMA: as many MFMAs as there are tile rows lie between, and 16 registers more did not fit.
    constexpr bool TWO = CT == 1 || L < 3;
    bf16x8 fa[TWO ? 2 : 1][L];
    float scale[CT];
    auto load_codes = [&](int slab, int stage, int q) __attribute__((always_inline)) {
      const unsigned so = slab < my_slabs ? (unsigned)(slab0 + slab) * 128u : kOutside;
      const unsigned v = !WHOLE && (slab0 + slab) * 8 + (cw ^ (4 * (q & 1))) >= blocks ? kOutside : vow[q];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_w, FK_LDS_PTR(lds + WBASE + stage * 4 * WSTAGE + wave * WSTAGE + q * 1024), 16, v, so, 0, 0);
    };
    auto load_scales = [&](int slab) __attribute__((always_inline)) {
      const int b0 = (slab0 + min(slab, my_slabs - 1)) * 8;
      if (WHOLE) next_sc = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs_s, vos, b0, 0));
      else next_sc = __builtin_bit_cast(u32x2, eight_scales(scales + vos, b0, blocks));
    };
    auto take_scales = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        if (CT == 2) {
          const u32x2 both = __builtin_amdgcn_permlane32_swap(next_sc[d], next_sc[d], false, false);      // the lower lanes' everywhere, the upper lanes' everywhere
          sc[0][d] = both[0];
          sc[CT - 1][d] = both[1];
        } else {
          sc[0][d] = next_sc[d];
        }
      }
    };
    const int swz = (frow >> 1) & 7;
    auto read_codes = [&](int stage, int j, int q) __attribute__((always_inline)) {
      w[j][q] = *(const u32x4 *)(lds + WBASE + stage * 4 * WSTAGE + wave * WSTAGE + (j * 32 + frow) * 128 + (((2 * q + h) ^ swz) << 4));
    };
    auto load_rows = [&](int step, int stage, int q) __attribute__((always_inline)) {
      const int k0 = slab0 * 256 + step * 64;
      const unsigned so = step < my_steps ? (unsigned)k0 * 2u : kOutside;
      const bool half = !WHOLE && k0 + 32 >= K;           // the second block of the step does not exist
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_a, FK_LDS_PTR(lds + stage * ASTAGE + (q * 4 + wave) * 1024), 16, half && ca >= 4 ? kOutside : voa[q], so, 0, 0);
    };
    // the scale of block 2 q + h of a slab, as a float
    auto scale_of = [&](u32x2 eight, int q) __attribute__((always_inline)) {
      const unsigned x = eight[q >> 1] >> (8 * h);
      return __uint_as_float(((q & 1) ? x << 7 : x << 23) & 0x7F800000u);
    };
    auto convert = [&](unsigned c, float by, int part) __attribute__((always_inline)) {
      return __builtin_bit_cast(unsigned, part == 0 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, by, 0) : part == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, by, 1)
                                                    : part == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, by, 2) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, by, 3));
    };
    unsigned first[4];          // this lane's fragment of each quarter of a step
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) first[ks] = frow * 128 + (((4 * h + ks) ^ ((frow >> 1) & 7)) << 4);

    // in an order in which the loop's count of younger loads holds from its first step on
    auto in_order = []() __attribute__((always_inline)) { loads_asked_for(); __builtin_amdgcn_sched_barrier(0); };
#pragma unroll
    for (int i = 0; i < SW; ++i)
#pragma unroll
      for (int q = 0; q < 4 * CT; ++q) load_codes(i, i, q);
    load_scales(0);
    in_order();
#pragma unroll
    for (int s = 0; s < SA; ++s) {
#pragma unroll
      for (int q = 0; q < L; ++q) load_rows(s, s, q);
      in_order();
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((SA - 1) * L));
    asm volatile("s_barrier" ::: "memory");
    take_scales();
#pragma unroll
    for (int i = 0; i < L; ++i) fa[0][i] = *(const bf16x8 *)(lds + first[0] + i * 4096);
#pragma unroll
    for (int j = 0; j < CT; ++j) read_codes(0, j, 0);
#pragma unroll
    for (int j = 0; j < CT; ++j) scale[j] = scale_of(sc[j], 0);
#pragma unroll
    for (int part = 0; part < 4; ++part) fb[0][part] = convert(w[0][0][0], scale[0], part);
    int stage = 0, code_stage = 0;              // of this step's rows, of this slab's codes
    // STEP: step of its slab.  A slab's first step reads the rest of its codes from LDS and, behind the barrier, asks for those that take their place.
    auto step_of = [&](auto which, int slab) __attribute__((always_inline)) {
      constexpr int STEP = decltype(which)::value;
      const int after = stage == SA - 1 ? 0 : stage + 1, next_code = code_stage == SW - 1 ? 0 : code_stage + 1;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        if (ks == 3) {
          // younger than the next step's rows: those of the step behind it, and, where they were asked for in the two steps before this
          // one, codes and scales
          __builtin_amdgcn_s_waitcnt(vmcnt_imm((SA - 2) * L + (STEP == 1 ? 4 * CT + (WHOLE ? 1 : 0) : 0)));
          asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
        // what is converted next: the other column tile's codes of this quarter, then this one's of the next
        const int word = (ks + 1) & 3;
        const unsigned char *const from = lds + first[word] + (ks == 3 ? after : stage) * ASTAGE;
#pragma unroll
        for (int s = 0; s < NMF; ++s) {
          const int j = s / L, i = s % L;
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fb[CT == 2 ? j : ks & 1]), fa[TWO ? ks & 1 : 0][i], acc[i][j], 0, 0, 0);
          if (TWO ? s < L : j == 1) fa[TWO ? (ks & 1) ^ 1 : 0][i] = *(const bf16x8 *)(from + i * 4096);
#pragma unroll
          for (int part = i * PER; part < i * PER + PER && part < 4; ++part) {
            if (CT == 2 && j == 0) {
              if (ks == 0 && part == 0) scale[CT - 1] = scale_of(sc[CT - 1], STEP);
              fb[1][part] = convert(w[CT - 1][STEP][ks], scale[CT - 1], part);
            } else {
              if (ks == 3 && part == 0) {
                if (STEP == 3) take_scales();
                scale[0] = scale_of(sc[0], (STEP + 1) & 3);
              }
              fb[CT == 2 ? 0 : (ks & 1) ^ 1][part] = convert(ks < 3 ? w[0][STEP][word] : w[0][(STEP + 1) & 3][0], scale[0], part);
            }
          }
          if (s == NMF - 1) {
            if (STEP == 0 && ks < 3) {
#pragma unroll
              for (int c = 0; c < CT; ++c) read_codes(code_stage, c, ks + 1);
            }
            if (STEP == 3 && ks == 2) {
#pragma unroll
              for (int c = 0; c < CT; ++c) read_codes(next_code, c, 0);
            }
          }
          if (STEP == 0 && ks == 3) {
#pragma unroll
            for (int q = s * 4 * CT / NMF; q < (s + 1) * 4 * CT / NMF; ++q) load_codes(slab + SW, code_stage, q);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        if (ks == 3) {
          if (STEP == 0) load_scales(slab + 1);
#pragma unroll
          for (int q = 0; q < L; ++q) load_rows(4 * slab + STEP + SA, stage, q);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      stage = after;
      if (STEP == 3) code_stage = next_code;
    };
    constexpr std::integral_constant<int, 0> s0;
    constexpr std::integral_constant<int, 1> s1;
    constexpr std::integral_constant<int, 2> s2;
    constexpr std::integral_constant<int, 3> s3;
    int slab = 0;
    for (; 4 * slab + 4 <= my_steps; ++slab) {
      step_of(s0, slab);
      step_of(s1, slab);
      step_of(s2, slab);
      step_of(s3, slab);
    }
    if (!WHOLE && 4 * slab < my_steps) {
      step_of(s0, slab);
      if (4 * slab + 1 < my_steps) step_of(s1, slab);
      if (4 * slab + 2 < my_steps) step_of(s2, slab);
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  };
  if (my_slabs <= 0) {}
  else if (TM == 1 || live == 1) multiply(std::integral_constant<int, 1>());
  else if (live == 2) multiply(std::integral_constant<int, TM < 2 ? 1 : 2>());
  else if (live == 3) multiply(std::integral_constant<int, TM < 3 ? 1 : 3>());
  else multiply(std::integral_constant<int, TM>());
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");                   // LDS is free
  using T = std::conditional_t<MODE == RM_STORE || SILU, bf16_t, float>;
  constexpr int G = SILU ? 2 * CT : 4 * CT;                                          // groups of 8 columns of this wavefront
  static_assert(4 * 32 * tile_pitch<T>(G) <= (int)sizeof(lds), "results of 32 rows of each wavefront");
  unsigned char *const mine = lds + wave * 32 * tile_pitch<T>(G);
  const int first = n0 + wave * 8 * G;
  T *const out = (T *)g.out + (MODE == RM_PARTIAL ? (size_t)split * g.split_stride : 0) + (size_t)row0 * g.ldo + first - g.n_begin;
  const bool wide = (((uintptr_t)g.out | ((MODE == RM_PARTIAL ? g.split_stride : 0) | (uint64_t)g.ldo) * sizeof(T)) & 15) == 0;
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    if (i * 32 >= valid) break;
    // SiLU*up: gate and up of a column are the same register of two tiles, or registers r and r + 8 of one
    auto value = [&](int v) __attribute__((always_inline)) {
      const f32x16 &t = acc[i][SILU ? 0 : v / 4];
      f32x4 x = {t[4 * (v % 4)], t[4 * (v % 4) + 1], t[4 * (v % 4) + 2], t[4 * (v % 4) + 3]};
      if (SILU) {
        const f32x16 &u = acc[i][CT - 1];
        const int at = CT == 2 ? 4 * v : 4 * (v & 1) + 8;
        // exp overflows to infinity and the quotient to 0 for a large negative gate
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = x[e] / (1.0f + __expf(-x[e])) * u[at + e];
      }
      return x;
    };
    store_tile<T, MODE == RM_ADD_F32, G>(mine, value, out + (int64_t)(i * 32) * g.ldo, g.ldo, valid - i * 32, n_end - first, wide);
  }
#endif
}

template <int BM, int CT, int MODE, bool GROUPED>
void launch_rows(hipStream_t s, RowsArgs g, int tile_slots) {
  g.tiles_n = MODE == RM_SILU ? (g.n_end - g.n_begin + 64 * CT - 1) / (64 * CT) : (g.n_end - g.n_begin + 128 * CT - 1) / (128 * CT);
  const int grid = GROUPED ? tile_slots * g.tiles_n : (tile_slots * g.tiles_n * g.splits + 7) / 8 * 8;
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
// MXFP4 rows x MXFP4 weights: 2 x 2 wavefronts.  K goes in pairs of slabs of 128: whole lines of 128 bytes of codes a row, straight into LDS, through
// a ring of mx_pairs() pairs (from the caches, lines of 128 bytes come at 34 TB/s over all compute units, pieces of 64 at 17).  Lane l supplies row
// l % 32 and, of the four quarters of 64 elements of a pair, block 2 q + l / 32: 16 bytes of codes and one scale.  Scales are fetched 16 bytes a row, for
// two pairs at once (a row per lane costs the vector caches a lookup per lane whatever its size), two pairs ahead, and handed on through LDS; those of a
// row's last blocks, where they are not 16, behind the loop.  Pipelined by hand like k_mx_rows: behind each MFMA one fragment read of the next quarter or
// one load.  The only barrier of a pair stands before its last quarter: by then everyone has read all of it, its place is filled again over the next
// quarters, and the next pair has landed.
// 2048 x 24576 x 4096: 106 to 110 us by card, 3.75 to 3.9 PFLOP/s.  The matrix units are busy in 43 % of the cycles, the loop without its loads takes 99 us and
// without its LDS reads 98, so none of the three alone is the bound; one workgroup a compute unit, in three rounds, overlaps neither its first loads nor its
// stores with anything.  Where K is no multiple of 256, rows begin inside a line and a piece of 128 bytes takes two of them: 333 x 4000, K = 12256, 25 us,
// K = 12288 20 (and 4 to 6 to add the two parts).
struct MxArgs {
  const unsigned char *A, *a_scales, *W, *w_scales;
  int M, N, K;
  int tiles_m, tiles_n, splits;
  void *out;
  int64_t ldo;
  size_t split_stride;
};
enum { XM_STORE, XM_STORE_F32, XM_PARTIAL };
// Pairs in LDS: what fits with one workgroup a compute unit.  (128 x 128 with two pairs and two workgroups a compute unit: 333 x 4096, K = 12288, 25.2 us
// instead of 23.1; 1024 x 4096, K = 4096, 17.3 instead of 15.3; 32 x 4096, K = 4096, 8.9 instead of 9.2.)
constexpr int mx_pairs(int bm) { return bm == 256 ? 2 : 4; }
constexpr int mx_lds(int bm, int bn) { return mx_pairs(bm) * (bm + bn) * 128 + 2 * (bm + bn) * 16; }

template <int BM, int BN, int MODE, bool WHOLE>      // WHOLE: K is a multiple of 512
__global__ __launch_bounds__(256, mx_lds(BM, BN) > 80 * 1024 ? 1 : 2) void k_mx_mx(MxArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int WM = BM / 2, WN = BN / 2, TM = WM / 32, TN = WN / 32, NMF = TM * TN, NF = TM + TN, IA = BM / 32, IB = BN / 32, ROWS = BM + BN, SI = ROWS / 256;
  // the loads of a pair are spread over SPREAD quarters, PART of them in each: the fewer pairs there are, the sooner they have to be asked for
  constexpr int R = mx_pairs(BM), L = IA + IB, SPREAD = R == 2 ? 2 : 4, PART = L / SPREAD, EVERY = NMF / PART;
  constexpr int ASTAGE = BM * 128, WSTAGE = BN * 128, WBASE = R * ASTAGE, SBASE = WBASE + R * WSTAGE;
  static_assert(NF <= NMF && PART <= NMF && NMF % PART == 0, "one fragment read and one load per MFMA at most");
  __shared__ __attribute__((aligned(1024))) unsigned char lds[mx_lds(BM, BN)];
  const int splits = g.splits, tiles_n = g.tiles_n, total = g.tiles_m * tiles_n * splits, per_xcd = (total + 7) / 8;
  const int item = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if ((int)(blockIdx.x / 8) >= per_xcd || item >= total) return;
  // tiles in groups of 8 tile rows, so that the panels of an XCD's range stay in its L2
  constexpr int GROUP = 8;
  const int split = item % splits, tile = item / splits;
  const int in_group = tile % (GROUP * tiles_n), first_m = tile / (GROUP * tiles_n) * GROUP, gsz = min(g.tiles_m - first_m, GROUP);
  const int m0 = (first_m + in_group % gsz) * BM, n0 = in_group / gsz * BN;
  const int M = g.M, N = g.N, K = g.K, blocks = K / 32, valid_m = min(BM, M - m0), valid_n = min(BN, N - n0);
  const int quads = (blocks + 15) / 16, per_split = (quads + splits - 1) / splits, slab0 = split * per_split * 4;
  const int slabs = min((blocks + 3) / 4 - slab0, per_split * 4);                    // of this workgroup
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = (wave >> 1) * WM, wn = (wave & 1) * WN, frow = lane & 31, h = lane >> 5;
  __amdgpu_buffer_rsrc_t rs_a = __builtin_amdgcn_make_buffer_rsrc((void *)(g.A + (size_t)m0 * (K / 2)), 0, (unsigned)valid_m * (unsigned)(K / 2), 0x00020000);
  __amdgpu_buffer_rsrc_t rs_w = __builtin_amdgcn_make_buffer_rsrc((void *)(g.W + (size_t)n0 * (K / 2)), 0, (unsigned)valid_n * (unsigned)(K / 2), 0x00020000);
  // An instruction fills 8 rows; lane l fetches chunk (block) (l % 8) ^ ((row / 2) % 8) of row l / 8, so that LDS reads spread over the banks.
  // Rows beyond the matrix lie outside the descriptors.  Behind a row's end come the next row's codes; their scales are taken as 0, 2^-127 on either side,
  // and 32 products of at most 36 times 2^-254 are nothing in fp32.
  const int chunk = (lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7);
  const unsigned vo = (unsigned)(wave * 8 + (lane >> 3)) * (unsigned)(K / 2) + chunk * 16, row_step = 32u * (unsigned)(K / 2);
  auto load = [&](int pair, int stage, int q) __attribute__((always_inline)) {          // q: 0 .. IA - 1 the rows, then the weights
    const unsigned so = 2 * pair < slabs ? (unsigned)(slab0 + 2 * pair) * 64u : kOutside;
    const int r = q < IA ? q : q - IA;
    const unsigned v = vo + r * row_step;
    if (q < IA) __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_a, FK_LDS_PTR(lds + stage * ASTAGE + (r * 4 + wave) * 1024), 16, v, so, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(rs_w, FK_LDS_PTR(lds + WBASE + stage * WSTAGE + (r * 4 + wave) * 1024), 16, v, so, 0, 0);
  };
  // scales of four slabs of SI rows per lane: rows of the tile, then of the weights; rows that do not exist take the last one's
  const unsigned char *srow[SI];
#pragma unroll
  for (int u = 0; u < SI; ++u) {
    const int r = (u * 4 + wave) * 64 + lane;
    srow[u] = r < BM ? g.a_scales + (size_t)(m0 + min(r, valid_m - 1)) * blocks : g.w_scales + (size_t)(n0 + min(r - BM, valid_n - 1)) * blocks;
  }
  u32x4 fetched[SI];
  // quads of which the row has all 16 blocks; behind the last of them it is not the quad's own scales that are fetched, and they count for nothing
  const int full = min(per_split, blocks / 16 - split * per_split);
  auto fetch_scales = [&](int quad) __attribute__((always_inline)) {
    const int b0 = min(slab0 * 4 + quad * 16, blocks - 16);
#pragma unroll
    for (int u = 0; u < SI; ++u) __builtin_memcpy(&fetched[u], srow[u] + b0, 16);
  };
  auto fetch_some_scales = [&](int quad) __attribute__((always_inline)) {      // any quad; slower, and many registers
    const int b0 = slab0 * 4 + quad * 16;
#pragma unroll
    for (int u = 0; u < SI; ++u) {
      const uint64_t lo = eight_scales(srow[u], b0, blocks), hi = eight_scales(srow[u], b0 + 8, blocks);
      fetched[u] = u32x4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
    }
  };
  auto hand_on_scales = [&](int quad) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < SI; ++u) *(u32x4 *)(lds + SBASE + (quad & 1) * ROWS * 16 + ((u * 4 + wave) * 64 + lane) * 16) = fetched[u];
  };
  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  // fragment s of a quarter in the order in which its MFMAs need them: W0, A0, W1 .. , A1 ..; the quarters differ in the chunk
  unsigned at_a[4], at_w[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const unsigned c = (unsigned)((2 * q + h) ^ ((frow >> 1) & 7)) << 4;
    at_a[q] = (wm + frow) * 128 + c;
    at_w[q] = WBASE + (wn + frow) * 128 + c;
  }
  u32x4 fa[2][TM], fw[2][TN];
  auto read = [&](int s, int q, int stage) __attribute__((always_inline)) {
    const int f = s == 0 ? TM : s == 1 ? 0 : s <= TN ? TM + s - 1 : s - TN;
    if (f < TM) fa[q & 1][f < TM ? f : 0] = *(const u32x4 *)(lds + at_a[q] + stage * ASTAGE + (f < TM ? f : 0) * 4096);
    else fw[q & 1][f < TM ? 0 : f - TM] = *(const u32x4 *)(lds + at_w[q] + stage * WSTAGE + (f < TM ? 0 : f - TM) * 4096);
  };
  // the four scales of a slab of every row, in two sets: byte 2 ks belongs to half ks once the upper lanes' are moved down by one
  unsigned ca[2][TM], cw[2][TN];
  auto read_scales = [&](int quad, int of_quad, int slot) __attribute__((always_inline)) {
    const unsigned char *from = lds + SBASE + (quad & 1) * ROWS * 16 + of_quad * 4;
#pragma unroll
    for (int i = 0; i < TM; ++i) ca[slot][i] = *(const unsigned *)(from + (wm + i * 32 + frow) * 16);
#pragma unroll
    for (int j = 0; j < TN; ++j) cw[slot][j] = *(const unsigned *)(from + (BM + wn + j * 32 + frow) * 16);
  };
  auto shift_scales = [&](int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TM; ++i) ca[slot][i] >>= 8 * h;
#pragma unroll
    for (int j = 0; j < TN; ++j) cw[slot][j] >>= 8 * h;
  };
  auto in_order = []() __attribute__((always_inline)) { loads_asked_for(); __builtin_amdgcn_sched_barrier(0); };
  if (slabs > 0) {
    if (WHOLE) fetch_scales(0);
    else fetch_some_scales(0);
    in_order();
#pragma unroll
    for (int p = 0; p < R; ++p) {
#pragma unroll
      for (int q = 0; q < (p < R - 1 ? L : PART); ++q) load(p, p, q);
      in_order();
    }
    hand_on_scales(0);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((R - 2) * L + PART));
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    read_scales(0, 0, 0);
#pragma unroll
    for (int s = 0; s < NF; ++s) read(s, 0, 0);
    // OF: slab of its quad of slabs, whose pairs lie at `stage` and behind it; MORE: scales of another quad are to be fetched
    auto slab_of = [&](auto which, int quad, auto more) __attribute__((always_inline)) {
      constexpr bool MORE = decltype(more)::value;
      constexpr int OF = decltype(which)::value, SLOT = OF & 1, NEXT = (OF + 1) & 3;
      const int pair = 2 * quad + OF / 2, stage = R == 2 ? OF / 2 : (2 * quad & (R - 1)) + OF / 2, after = OF < 2 ? stage + 1 : R == 2 ? 0 : (stage + 1) & (R - 1);
      shift_scales(SLOT);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        constexpr int FIRST = 2 * (OF & 1);
        const int q = FIRST + ks;              // of the pair
        if (q == 3) {
          if (MORE && OF == 3) hand_on_scales(quad + 1);
          // the next pair has landed: younger are those of the pairs behind it (and scales, which are not counted)
          __builtin_amdgcn_s_waitcnt(vmcnt_imm((R - 2) * L));
          asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
          if (MORE && OF == 1) { fetch_scales(quad + 1); in_order(); }
        }
        if (ks == 1) read_scales(OF == 3 ? quad + 1 : quad, NEXT, SLOT ^ 1);
#pragma unroll
        for (int s = 0; s < NMF; ++s) {
          const int i = s / TN, j = s % TN;
          const i32x8 a = {(int)fa[ks][i][0], (int)fa[ks][i][1], (int)fa[ks][i][2], (int)fa[ks][i][3], 0, 0, 0, 0};
          const i32x8 b = {(int)fw[ks][j][0], (int)fw[ks][j][1], (int)fw[ks][j][2], (int)fw[ks][j][3], 0, 0, 0, 0};
          if (ks == 0) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, acc[i][j], 4, 4, 0, (int)cw[SLOT][j], 0, (int)ca[SLOT][i]);
          else acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, acc[i][j], 4, 4, 2, (int)cw[SLOT][j], 2, (int)ca[SLOT][i]);
          if (s < NF) read(s, (q + 1) & 3, q == 3 ? after : stage);
          // spread: in a burst the loads hold up the MFMAs behind them for as long as the address unit takes
          if (s % EVERY == EVERY - 1) {
            if (q == 3) load(pair + R, stage, s / EVERY);
            else if (q + 1 < SPREAD) load(pair + R - 1, R == 2 ? stage ^ 1 : (stage + R - 1) & (R - 1), (q + 1) * PART + s / EVERY);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    constexpr std::integral_constant<int, 0> s0;
    constexpr std::integral_constant<int, 1> s1;
    constexpr std::integral_constant<int, 2> s2;
    constexpr std::integral_constant<int, 3> s3;
    constexpr std::integral_constant<bool, true> yes;
    constexpr std::integral_constant<bool, false> no;
    int quad = 0;
    for (; quad < full; ++quad) {
      slab_of(s0, quad, yes);
      slab_of(s1, quad, yes);
      slab_of(s2, quad, yes);
      slab_of(s3, quad, yes);
    }
    if (!WHOLE && 4 * quad < slabs) {
      if (quad > 0) {
        fetch_some_scales(quad);
        hand_on_scales(quad);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        read_scales(quad, 0, 0);
      }
      slab_of(s0, quad, no);
      if (4 * quad + 1 < slabs) slab_of(s1, quad, no);
      if (4 * quad + 2 < slabs) slab_of(s2, quad, no);
      if (4 * quad + 3 < slabs) slab_of(s3, quad, no);
    }
  }
  __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");                   // LDS is free
  using T = std::conditional_t<MODE == XM_STORE, bf16_t, float>;
  static_assert(4 * 32 * tile_pitch<T>(4 * TN) <= (int)sizeof(lds), "results of 32 rows of each wavefront");
  unsigned char *const mine = lds + wave * 32 * tile_pitch<T>(4 * TN);
  T *const out = (T *)g.out + (MODE == XM_PARTIAL ? (size_t)split * g.split_stride : 0) + (size_t)(m0 + wm) * g.ldo + n0 + wn;
  const bool wide = (((uintptr_t)g.out | ((MODE == XM_PARTIAL ? g.split_stride : 0) | (uint64_t)g.ldo) * sizeof(T)) & 15) == 0;
#pragma unroll
  for (int i = 0; i < TM; ++i)
    store_tile<T, false, 4 * TN>(mine, [&](int v) __attribute__((always_inline)) { const f32x16 &t = acc[i][v / 4]; return f32x4{t[4 * (v % 4)], t[4 * (v % 4) + 1], t[4 * (v % 4) + 2], t[4 * (v % 4) + 3]}; }, out + (int64_t)(i * 32) * g.ldo, g.ldo, valid_m - wm - i * 32, valid_n - wn, wide);
#endif
}

template <int BM, int BN, int MODE>
void launch_mx(hipStream_t s, const MxArgs &g) {
  const int grid = (g.tiles_m * g.tiles_n * g.splits + 7) / 8 * 8;
  if (g.K % 512 == 0 && g.K > 0) k_mx_mx<BM, BN, MODE, true><<<grid, 256, 0, s>>>(g);
  else k_mx_mx<BM, BN, MODE, false><<<grid, 256, 0, s>>>(g);
}
template <int BM, int BN>
void launch_mx(hipStream_t s, int mode, MxArgs g) {
  g.tiles_m = (g.M + BM - 1) / BM;
  g.tiles_n = (g.N + BN - 1) / BN;
  if (mode == XM_STORE) launch_mx<BM, BN, XM_STORE>(s, g);
  else if (mode == XM_STORE_F32) launch_mx<BM, BN, XM_STORE_F32>(s, g);
  else launch_mx<BM, BN, XM_PARTIAL>(s, g);
}

// ---------------------------------------------------------------------------------------------
// Adds the parts of a cut K in part order and does the epilogue.  A thread takes V neighbouring columns of a row (four where the rows of all operands
// are 16-byte aligned), and all its parts are asked for before the first is added, four at a time.
template <int EPI, int V>
__global__ __launch_bounds__(256) void k_mx_reduce(const float *__restrict__ part, int splits, size_t stride, Rows rows, int n, void *out, int64_t ldo) {
  typedef float fv __attribute__((ext_vector_type(V)));
  const int M = rows.count ? min(*rows.count, rows.cap) : rows.cap, cols = EPI == MX_SILU_MUL ? n / 2 : n;
  const int col = (blockIdx.x * 256 + threadIdx.x) * V;
  if (col >= cols) return;
  for (int row = blockIdx.y; row < M; row += gridDim.y) {
    const float *p = part + (size_t)row * n + col;
    fv v = 0.f, u = 0.f;
    for (int k0 = 0; k0 < splits; k0 += 4) {
      fv a[4], b[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        a[k] = k0 + k < splits ? *(const fv *)(p + (size_t)(k0 + k) * stride) : (fv)0.f;
        if (EPI == MX_SILU_MUL) b[k] = k0 + k < splits ? *(const fv *)(p + (size_t)(k0 + k) * stride + n / 2) : (fv)0.f;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v += a[k];
        if (EPI == MX_SILU_MUL) u += b[k];
      }
    }
    const size_t at = (size_t)row * ldo + col;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (EPI == MX_STORE) ((bf16_t *)out)[at + i] = (bf16_t)v[i];
      else if (EPI == MX_STORE_F32) ((float *)out)[at + i] = v[i];
      else if (EPI == MX_ADD_F32) ((float *)out)[at + i] += v[i];
      else ((bf16_t *)out)[at + i] = (bf16_t)(v[i] / (1.0f + __expf(-v[i])) * u[i]);
    }
  }
}

template <int V> void launch_reduce(hipStream_t s, int epi, const float *part, int splits, size_t stride, Rows rows, int n, void *out, int64_t ldo) {
  const int cols = epi == MX_SILU_MUL ? n / 2 : n;
  const dim3 grid((cols + 256 * V - 1) / (256 * V), std::min(rows.cap, 32768));
  if (epi == MX_STORE) k_mx_reduce<MX_STORE, V><<<grid, 256, 0, s>>>(part, splits, stride, rows, n, out, ldo);
  else if (epi == MX_STORE_F32) k_mx_reduce<MX_STORE_F32, V><<<grid, 256, 0, s>>>(part, splits, stride, rows, n, out, ldo);
  else if (epi == MX_ADD_F32) k_mx_reduce<MX_ADD_F32, V><<<grid, 256, 0, s>>>(part, splits, stride, rows, n, out, ldo);
  else k_mx_reduce<MX_SILU_MUL, V><<<grid, 256, 0, s>>>(part, splits, stride, rows, n, out, ldo);
}
void launch_reduce(hipStream_t s, int epi, const float *part, int splits, size_t stride, Rows rows, int n, void *out, int64_t ldo) {
  // the parts' rows are n apart, and so are the parts' starts rows.cap * n: both multiples of four where n (with SiLU*up half of it) is
  if (n % (epi == MX_SILU_MUL ? 8 : 4) == 0 && ((uintptr_t)part & 15) == 0) launch_reduce<4>(s, epi, part, splits, stride, rows, n, out, ldo);
  else launch_reduce<1>(s, epi, part, splits, stride, rows, n, out, ldo);
}

// parts with no unit of K left over are dropped
int whole_parts(int parts, int units) { const int per = (units + parts - 1) / parts; return (units + per - 1) / per; }

// Tile and parts of K with the least estimated time.  Measured on 15 problems of 8 to 2048 rows, 2048 to 24576 columns and K of 2048 to 12288, every
// tile with up to 16 parts.  A unit of K (256; with both operands in MXFP4 512) takes a workgroup `base` us alone and `first` more when all 256 compute
// units have one; a second on some of them makes it `second`, and `more` for each further 256; beyond per_cu of them rounds follow one another.  A launch
// costs 3 us, adding parts 2.5 us and 8 bytes an output and part at 4.5 TB/s.  (333 rows x 4096, K = 4096, MXFP4 rows: 12.5 us in one part, 22 in five,
// which fill the chip; K = 12288: 27.5 in one, 23.1 in two, 30 in three.  1024 rows, K = 4096: 128 x 128 15.3, 256 x 256 28.5; 2048 rows x 6144: 45.5 and
// 35.3.  bf16 rows: 8 x 24576 32 x 128 17.4, 128 x 128 17.9; 1024 x 4096 128 x 128 36.6, 128 x 256 46.9; 333 x 4096, K = 12288, 128 x 128: 50.3 in two,
// 49.5 in five, 128 x 256 49.3 in five.)  Its choices are the fastest of those or within 4 % of it.
struct Variant { int bm, bn, per_cu; float base, first, second, more; };
constexpr Variant kRowVariants[] = {{32, 128, 3, 0.8f, 0.45f, 1.3f, 0.7f}, {128, 128, 2, 1.4f, 0.9f, 3.0f, 0.8f}, {128, 256, 2, 2.8f, 0.9f, 5.2f, 1.5f}};
constexpr Variant kMxVariants[] = {{128, 128, 1, 0.85f, 0.6f, 0.f, 0.f}, {256, 256, 1, 2.6f, 1.3f, 0.f, 0.f}};
float unit_us(const Variant &v, int64_t groups) {
  const int64_t round = 256 * v.per_cu, rounds = (groups - 1) / round, left = groups - rounds * round;
  auto one = [&](int64_t n) { return n <= 256 ? v.base + v.first * (float)n / 256.f : v.second + v.more * (float)(n - 256) / 256.f; };
  return (float)rounds * one(round) + one(left);
}
struct Shape { int bm, bn, splits; };
Shape shape_of(int rows, int n, int k, bool a_mx) {
  const int units = std::max(1, a_mx ? (k / 32 + 15) / 16 : (k / 32 + 7) / 8);
  Shape best{0, 0, 1};
  float least = 0.f;
  for (const Variant *v = a_mx ? kMxVariants : kRowVariants, *end = a_mx ? std::end(kMxVariants) : std::end(kRowVariants); v != end; ++v) {
    const int tiles_m = (rows + v->bm - 1) / v->bm;
    const int64_t tiles = (int64_t)tiles_m * ((n + v->bn - 1) / v->bn);
    if (tiles > kMaxGroups - 8) continue;
    // tile rows of 32 that hold no rows are skipped
    const float live = a_mx || v->bm == 32 ? 1.f : 0.4f + 0.6f * (float)((rows + 31) / 32) / (float)(tiles_m * v->bm / 32);
    for (int parts = 1; parts <= std::min(units, 16); ++parts) {
      if (whole_parts(parts, units) != parts || (parts > 1 && tiles * parts > 1024)) continue;
      const float us = 3.f + live * unit_us(*v, tiles * parts) * (float)((units + parts - 1) / parts) + (parts > 1 ? 2.5f + (float)parts * (float)rows * (float)n * (8.f / 4.5e6f) : 0.f);
      if (!best.bm || us < least) { best = {v->bm, v->bn, parts}; least = us; }
    }
  }
  return best;
}

}  // namespace

size_t mx_gemm_scratch(int rows, int n, int k, bool a_mx) {
  const Shape p = shape_of(rows, n, k, a_mx);
  return p.splits > 1 ? (size_t)p.splits * rows * n * 4 : 0;
}

void mx_gemm(hipStream_t s, const void *a, const void *a_scales, int64_t lda, focus_mx w, int n, int k, Rows rows, int epilogue, void *out, int64_t ldo, Scratch scratch) {
  if (rows.cap <= 0 || n <= 0) return;
  const bool a_mx = a_scales != nullptr;
  Shape p = shape_of(rows.expected(), n, k, a_mx);
  // the grid has room for rows.cap, however few are expected
  if (!a_mx && (int64_t)((rows.cap + p.bm - 1) / p.bm) * ((n + p.bn - 1) / p.bn) * p.splits > kMaxGroups - 8) p = {128, 128, 1};
  const size_t stride = (size_t)rows.cap * n;
  const int units = a_mx ? (k / 32 + 15) / 16 : (k / 32 + 7) / 8;
  if (p.splits > 1) p.splits = whole_parts((int)std::max<size_t>(1, std::min<size_t>(p.splits, scratch.ptr ? scratch.bytes / (stride * 4) : 0)), units);
  const bool parts = p.splits > 1;
  if (a_mx) {
    MxArgs g{(const unsigned char *)a, (const unsigned char *)a_scales, (const unsigned char *)w.codes, (const unsigned char *)w.scales, rows.cap, n, k, 0, 0, p.splits,
             parts ? scratch.ptr : out, parts ? n : ldo, stride};
    const int mode = parts ? XM_PARTIAL : epilogue == MX_STORE ? XM_STORE : XM_STORE_F32;
    if (p.bm == 256) launch_mx<256, 256>(s, mode, g);
    else launch_mx<128, 128>(s, mode, g);
  } else {
    RowsArgs g{};
    g.A = (const bf16_t *)a; g.lda = lda; g.codes = (const unsigned char *)w.codes; g.scales = (const unsigned char *)w.scales; g.N = n; g.K = k; g.rows = rows; g.n_end = epilogue == MX_SILU_MUL && !parts ? n / 2 : n;
    g.splits = p.splits; g.split_stride = stride; g.out = parts ? scratch.ptr : out; g.ldo = parts ? n : ldo;
    const int mode = parts ? RM_PARTIAL : epilogue == MX_STORE ? RM_STORE : epilogue == MX_STORE_F32 ? RM_STORE_F32 : epilogue == MX_ADD_F32 ? RM_ADD_F32 : RM_SILU;
    if (p.bm == 32) launch_rows<32, 1>(s, mode, g, (rows.cap + 31) / 32);
    else if (p.bn == 256) launch_rows<128, 2>(s, mode, g, (rows.cap + 127) / 128);
    else launch_rows<128, 1>(s, mode, g, (rows.cap + 127) / 128);
  }
  if (parts) launch_reduce(s, epilogue, (const float *)scratch.ptr, p.splits, stride, rows, n, out, ldo);
}

// Tiles of 32 x 128 for up to kMxFewRows rows per expert on average: more workgroups, whose loads of codes few others share (whole operator in us, 32-row
// tiles / 128-row ones: 256 experts, 2048 -> 512, 1 row an expert 75.8 / 79.2, 4 rows 108 / 105, 8 118 / 115, 16 135 / 126, 32 172 / 154; 160 experts,
// 2560 -> 320, 4 rows 66 / 74, 7 rows 79 / 78).  Above, 128 x 256 where there may be kMxWide of them, 128 x 128 where the wide ones would leave compute
// units idle (128 x 256 / 128 x 128: 256 experts, 2048 -> 512, 64 rows 197 / 219; 8 experts, 2560 -> 1408, 64 rows 60 / 43, 256 rows 84 / 79, 1024 rows
// 209 / 215; 32 experts, 1024 -> 768, 128 rows 53 / 49).
constexpr int kMxWide = 512;
template <int MODE>
static void launch_grouped(hipStream_t s, const RowsArgs &a, const MxExperts &m) {
  const int slots = mx_tile_slots(m.rows.cap, m.k, m.n_experts, m.tile_rows);
  if (m.tile_rows == 32) launch_rows<32, 1, MODE, true>(s, a, slots);
  else if ((int64_t)mx_tile_slots(m.rows.expected(), m.k, m.n_experts, 128) * (((MODE == RM_SILU ? 2 : 1) * (a.n_end - a.n_begin) + 255) / 256) >= kMxWide) launch_rows<128, 2, MODE, true>(s, a, slots);
  else launch_rows<128, 1, MODE, true>(s, a, slots);
}

// The activations are rounded to bf16, the operand type of the matrix instruction that multiplies them with the down matrices (in fp32 they would be two bf16
// operands, and the second product twice as long).  1024 rows through 8 of 64 experts, 2048 -> 512, against 64 bits: relative error 1.7e-3 with fp32 results (1.5e-5
// against 64 bits with the same rounding), 2.3e-3 with bf16 results, whose own rounding alone gives 1.7e-3.
void mx_up(hipStream_t s, const MxExperts &m) {
  if (m.rows.cap <= 0) return;
  RowsArgs a{};
  a.A = (const bf16_t *)m.x; a.lda = m.ldx; a.src = m.arow; a.a_bytes = (unsigned)(((int64_t)(m.rows.cap - 1) * m.ldx + m.hidden) * 2);
  a.codes = (const unsigned char *)m.gate_up.codes; a.scales = (const unsigned char *)m.gate_up.scales;
  a.N = 2 * m.ffn; a.n_end = m.ffn; a.K = m.hidden; a.tiles = m.tiles; a.n_tiles = m.n_tiles; a.splits = 1; a.out = m.act; a.ldo = m.ffn;
  launch_grouped<RM_SILU>(s, a, m);
}

// ---------------------------------------------------------------------------------------------
// Entries sorted by expert.  Which of a workgroup's entries of one expert comes first is left to the order of its LDS atomics: a row's sums do
// not depend on its place in a tile.
namespace {
constexpr int kChunk = 1024;      // entries of a workgroup; at least kMxMaxExperts
// Up to so many chunks every workgroup of the one launch counts all entries; from there on a launch of its own counts them chunk by chunk first
// (the quadratic counting of 16 chunks takes 3 us, the second launch 5).
constexpr int kCountAll = 16;

__global__ __launch_bounds__(kChunk) void k_mx_count(MxExperts a) {
  __shared__ int cnt[kMxMaxExperts];
  const int E = a.n_experts, tid = threadIdx.x, M = a.rows.count ? min(*a.rows.count, a.rows.cap) : a.rows.cap, n = M * a.k;
  if (tid < E) cnt[tid] = 0;
  __syncthreads();
  const int i = blockIdx.x * kChunk + tid;
  if (i < n) {
    const int e = a.experts[i];
    if (e >= 0 && e < E) atomicAdd(&cnt[e], 1);
  }
  __syncthreads();
  if (tid < E) a.hist[(size_t)blockIdx.x * E + tid] = cnt[tid];
}

// Thread e < E knows how many entries of expert e there are, in all and in the chunks before this workgroup's.  The tiles are listed by falling
// number of tile rows of 32: full ones, then those of three, two and one, each in the order of the experts.
template <bool COUNTED>
__global__ __launch_bounds__(kChunk) void k_mx_place(MxExperts a, int chunks, int tile_slots) {
  __shared__ int next[kMxMaxExperts];
  __shared__ uint64_t wide[kChunk / 64];
  __shared__ unsigned narrow[kChunk / 64];
  const int E = a.n_experts, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, me = blockIdx.x;
  const int M = a.rows.count ? min(*a.rows.count, a.rows.cap) : a.rows.cap, n = M * a.k;
  int before = 0, all = 0, own = -1;
  constexpr int U = 16;
  static_assert(kCountAll <= U, "one round of loads when nothing was counted");
  if (COUNTED) {
    if (tid < E)
      for (int c0 = 0; c0 < chunks; c0 += U) {
        int v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = c0 + u < chunks ? a.hist[(size_t)(c0 + u) * E + tid] : 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          before += c0 + u < me ? v[u] : 0;
          all += v[u];
        }
      }
    if (me * kChunk + tid < n) own = a.experts[me * kChunk + tid];
  } else {
    int v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = u < chunks && u * kChunk + tid < n ? a.experts[u * kChunk + tid] : -1;
    if (tid < E) next[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u == me) {
        own = v[u];
        __syncthreads();
        if (tid < E) before = next[tid];
        __syncthreads();
      }
      if (v[u] >= 0 && v[u] < E) atomicAdd(&next[v[u]], 1);
    }
    __syncthreads();
    if (tid < E) all = next[tid];
  }
  // exclusive sums over the experts of rows and full tiles, and of tiles of three, two and one tile rows (10 bits each)
  const int T = a.tile_rows, full = all / T, rest = (all % T + 31) / 32 % (T / 32), whole = full + (all % T > T - 32);
  const uint64_t w0 = ((uint64_t)whole << 32) | (unsigned)all;
  const unsigned n0 = rest ? 1u << (10 * (3 - rest)) : 0u;
  uint64_t w = w0;
  unsigned q = n0;
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t wo = __shfl_up((unsigned long long)w, d);
    const unsigned qo = __shfl_up(q, d);
    if (lane >= d) { w += wo; q += qo; }
  }
  if (lane == 63) { wide[wave] = w; narrow[wave] = q; }
  __syncthreads();
  uint64_t w_all = 0;
  unsigned q_all = 0;
  w -= w0;
  q -= n0;
  for (int i = 0; i < kMxMaxExperts / 64; ++i) {       // experts are the first threads
    if (i < wave) { w += wide[i]; q += narrow[i]; }
    w_all += wide[i];
    q_all += narrow[i];
  }
  const int first = (int)(unsigned)w;
  if (tid < E) {
    next[tid] = first + before;
    if (me == 0) {
      int t = (int)(w >> 32);
      for (int m = 0; m < whole; ++m, ++t)
        if (t < tile_slots) a.tiles[t] = make_int2(first + m * T, tid | min(T, all - m * T) << 16);
      if (rest) {
        t = (int)(w_all >> 32);
        for (int r = 3; r > rest; --r) t += q_all >> (10 * (3 - r)) & 1023;
        t += q >> (10 * (3 - rest)) & 1023;
        if (t < tile_slots) a.tiles[t] = make_int2(first + full * T, tid | (all - full * T) << 16);
      }
    }
  }
  if (me == 0 && tid == 0) {
    int t = (int)(w_all >> 32);
    for (int r = 0; r < 3; ++r) t += q_all >> (10 * r) & 1023;
    *a.n_tiles = min(t, tile_slots);
  }
  __syncthreads();
  const int i = me * kChunk + tid;
  if (i < n) {
    int p = -1;
    if (own >= 0 && own < E) {
      p = atomicAdd(&next[own], 1);
      a.arow[p] = i / a.k;
    }
    a.pos[i] = p;
  }
}

// out[row] (+)= sum_j weight_j y[pos_j], j ascending, for the columns from c0 on that y holds (cols of them), four to a thread.  Eight products are asked
// for at once: one after the other, each behind its place in the list, 8 rows take 4.4 us instead of 3.9.  Many rows are bound by the reads of y either way:
// 2048 rows of 8 products, 2048 columns, 134 MB, 23 us (5.8 TB/s, from the memory-side cache).
template <typename T, bool ADD>
__global__ __launch_bounds__(256) void k_mx_combine(MxExperts a, int c0, int cols) {
  const int row = blockIdx.x, k = a.k;
  if (a.rows.count && row >= *a.rows.count) return;
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * 4;
  if (c >= cols) return;
  const int32_t *const pos = a.pos + (size_t)row * k;
  const float *const weights = a.weights + (size_t)row * k;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < k; j0 += 8) {
    int p[8];
    float w[8];
    float4 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      p[j] = j0 + j < k ? pos[j0 + j] : -1;
      w[j] = j0 + j < k ? weights[j0 + j] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = *(const float4 *)(a.y + (size_t)max(p[j], 0) * cols + c);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (p[j] >= 0) { acc[0] += w[j] * v[j].x; acc[1] += w[j] * v[j].y; acc[2] += w[j] * v[j].z; acc[3] += w[j] * v[j].w; }
  }
  T *o = (T *)a.out + (size_t)row * a.ldo + c0 + c;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = ADD ? (T)((float)o[i] + acc[i]) : (T)acc[i];
}
}  // namespace

int mx_tile_rows(int rows, int k, int n_experts) { return rows * k <= kMxFewRows * std::min(rows * k, n_experts) ? 32 : 128; }
// Row tiles there can be, rounded up to the eight XCDs that take them in turn.
int mx_tile_slots(int rows, int k, int n_experts, int tile_rows) { return (rows * k / tile_rows + std::min(rows * k, n_experts) + 7) / 8 * 8; }
// Columns of a slice of the second product: a multiple of 256.
static int mx_slice(int rows, int k, int hidden) {
  const int64_t fit = kMxSliceBytes / ((int64_t)rows * k * 4) / 256 * 256;
  return fit >= hidden ? hidden : (int)std::max<int64_t>(fit, 256);
}
int mx_chunks(int rows, int k) { return (rows * k + kChunk - 1) / kChunk; }

// Lays the work buffers out from `base`; returns their size.
static size_t lay(MxExperts &a, char *base, int rows) {
  const size_t ent = (size_t)rows * a.k;
  size_t at = 0;
  auto take = [&](size_t bytes) { char *p = base + at; at += (bytes + 255) & ~(size_t)255; return p; };
  a.hist = (int32_t *)take((size_t)mx_chunks(rows, a.k) * a.n_experts * 4);
  a.tile_rows = mx_tile_rows(rows, a.k, a.n_experts);
  a.tiles = (int2 *)take((size_t)mx_tile_slots(rows, a.k, a.n_experts, a.tile_rows) * 8);
  a.n_tiles = (int32_t *)take(4);
  a.pos = (int32_t *)take(ent * 4);
  a.arow = (int32_t *)take(ent * 4);
  a.act = take(ent * a.ffn * 2);
  a.y = (float *)take(ent * std::min(a.hidden, mx_slice(std::max(1, rows), a.k, a.hidden)) * 4);
  return at;
}
size_t mx_experts_bytes(int n_experts, int hidden, int ffn, int n_rows, int k) {
  MxExperts a{};
  a.n_experts = n_experts; a.hidden = hidden; a.ffn = ffn; a.k = k;
  return lay(a, nullptr, n_rows);
}
void lay_mx_experts(MxExperts &a, void *workspace) { lay(a, (char *)workspace, a.rows.cap); }

void mx_group(hipStream_t s, const MxExperts &a) {
  if (a.rows.cap <= 0) return;
  const int chunks = mx_chunks(a.rows.cap, a.k), slots = mx_tile_slots(a.rows.cap, a.k, a.n_experts, a.tile_rows);
  if (chunks <= kCountAll) {
    k_mx_place<false><<<chunks, kChunk, 0, s>>>(a, chunks, slots);
  } else {
    k_mx_count<<<chunks, kChunk, 0, s>>>(a);
    k_mx_place<true><<<chunks, kChunk, 0, s>>>(a, chunks, slots);
  }
}

// The second product and the weighted sums, so many columns at a time that the fp32 products of a slice stay in the memory-side cache (256 MB) between the
// two launches, and the next slice's go where they were: 8192 rows through 8 of 256 experts each, 512 -> 2048, 537 MB of products, in four slices 4 x (60 + 23) us; in one the
// sums alone took 137 instead of 91.
void mx_down(hipStream_t s, const MxExperts &m) {
  if (m.rows.cap <= 0) return;
  RowsArgs a{};
  a.A = (const bf16_t *)m.act; a.lda = m.ffn;
  a.codes = (const unsigned char *)m.down.codes; a.scales = (const unsigned char *)m.down.scales;
  a.N = m.hidden; a.K = m.ffn; a.tiles = m.tiles; a.n_tiles = m.n_tiles; a.splits = 1; a.out = m.y;
  const int slice = mx_slice(m.rows.cap, m.k, m.hidden);
  for (int c0 = 0; c0 < m.hidden; c0 += slice) {
    const int cols = std::min(slice, m.hidden - c0);
    a.n_begin = c0; a.n_end = c0 + cols; a.ldo = cols;
    launch_grouped<RM_STORE_F32>(s, a, m);
    const int threads = std::min(256, (cols / 4 + 63) / 64 * 64);
    const dim3 grid(m.rows.cap, (cols / 4 + threads - 1) / threads);
    if (m.out_type == FOCUS_BF16) k_mx_combine<bf16_t, false><<<grid, threads, 0, s>>>(m, c0, cols);
    else if (m.add) k_mx_combine<float, true><<<grid, threads, 0, s>>>(m, c0, cols);
    else k_mx_combine<float, false><<<grid, threads, 0, s>>>(m, c0, cols);
  }
}

}  // namespace fk
