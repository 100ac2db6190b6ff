// Conversion of rows to microscaled 4-bit floats (MXFP4) and back.  Both are bound by memory: 2 or 4 bytes an element on one side, 17/32 on the other.
// 65536 x 2048 bf16: 71 to 74 us in, 63 us out, 340 MB each, 4.6 to 5.4 TB/s, what a large copy reaches (5.0); 333 x 1000 fp32: 2.7 us each, a launch.
#include "focus_mx.h"

namespace fk {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// A thread converts 8 neighbours (16 or 32 bytes in one or two accesses, 4 bytes of codes), four neighbouring threads a block of 32, whose largest exponent
// they find by two lane exchanges; the scale needs no logarithm: it is the exponent field less two.  Chunk i of the matrix
// lies in row i / per_row; per_row is a multiple of 4, so the four threads of a block are lanes of one quad.
struct Chunks {
  int64_t total, per_row;
  int cols;                // of a row
  int64_t ldx;
  bool one_row;            // the matrix is one long run: no division
};
__device__ __forceinline__ void locate(const Chunks &g, int64_t i, int64_t &row, int64_t &col) {
  if (g.one_row) { row = 0; col = i * 8; return; }
  row = g.total < (1ll << 31) ? (int64_t)((unsigned)i / (unsigned)g.per_row) : i / g.per_row;
  col = (i - row * g.per_row) * 8;
}

// 8 elements as fp32 bits' worth of data: bf16 stays packed
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  u32x4 v;
  __device__ void load(const bf16_t *p) { v = *(const u32x4 *)p; }
  __device__ void load_some(const bf16_t *p, int n) {
    const unsigned short *q = (const unsigned short *)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (2 * i < n ? q[2 * i] : 0u) | (2 * i + 1 < n ? (unsigned)q[2 * i + 1] << 16 : 0u);
  }
  __device__ unsigned exponent() const {       // largest biased exponent
    u16x2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7F807F80u));
    return (unsigned)(m[0] > m[1] ? m[0] : m[1]) >> 7;
  }
  template <int B> __device__ unsigned convert(unsigned old, float scale) const {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(old, __builtin_bit_cast(bf16x2, (unsigned)v[B]), scale, B);
  }
};
template <> struct Eight<float> {
  u32x4 v[2];
  __device__ void load(const float *p) { v[0] = ((const u32x4 *)p)[0]; v[1] = ((const u32x4 *)p)[1]; }
  __device__ void load_some(const float *p, int n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = i < n ? ((const unsigned *)p)[i] : 0u;
  }
  __device__ unsigned exponent() const {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, v[i >> 2][i & 3] & 0x7F800000u);
    return m >> 23;
  }
  template <int B> __device__ unsigned convert(unsigned old, float scale) const {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(old, __uint_as_float(v[B >> 1][2 * (B & 1)]), __uint_as_float(v[B >> 1][2 * (B & 1) + 1]), scale, B);
  }
};

template <int CTRL> __device__ __forceinline__ unsigned quad_max(unsigned v) {
  return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false));
}

// VEC: whole chunks may be read 16 bytes at a time
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_mx_quantize(Chunks g, const T *__restrict__ x, unsigned *__restrict__ codes, unsigned char *__restrict__ scales) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= g.total) return;
  int64_t row, col;
  locate(g, i, row, col);
  const T *p = x + row * g.ldx + col;
  Eight<T> e;
  const int64_t left = g.one_row ? 8 : g.cols - col;
  if (VEC && left >= 8) e.load(p);
  else e.load_some(p, left < 0 ? 0 : left < 8 ? (int)left : 8);
  unsigned ex = quad_max<0x4E>(quad_max<0xB1>(e.exponent()));
  // floor(log2(max)) - 2 = exponent field - 127 - 2
  const unsigned s = ex == 255 ? 255 : ex > 2 ? ex - 2 : 0;
  const float scale = __uint_as_float(s << 23);
  unsigned c = e.template convert<0>(0, scale);
  c = e.template convert<1>(c, scale);
  c = e.template convert<2>(c, scale);
  c = e.template convert<3>(c, scale);
  codes[i] = s == 255 ? 0 : c;
  if ((i & 3) == 0) scales[i >> 2] = (unsigned char)s;
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_mx_dequantize(Chunks g, const unsigned *__restrict__ codes, const unsigned char *__restrict__ scales, T *__restrict__ x) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= g.total) return;
  int64_t row, col;
  locate(g, i, row, col);
  T *p = x + row * g.ldx + col;
  const unsigned c = codes[i], s = scales[i >> 2];
  float v[8];
  const float scale = __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7FC00000u : s << 23);
  f32x2 q;
  q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 0); v[0] = q[0] * scale; v[1] = q[1] * scale;
  q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 1); v[2] = q[0] * scale; v[3] = q[1] * scale;
  q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 2); v[4] = q[0] * scale; v[5] = q[1] * scale;
  q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.f, 3); v[6] = q[0] * scale; v[7] = q[1] * scale;
  const int64_t left = g.one_row ? 8 : g.cols - col;
  if (VEC && left >= 8) {
    if (sizeof(T) == 4) {
      ((float4 *)p)[0] = make_float4(v[0], v[1], v[2], v[3]);
      ((float4 *)p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      u32x4 o;
#pragma unroll
      for (int j = 0; j < 4; ++j) { const bf16x2 b = {(__bf16)v[2 * j], (__bf16)v[2 * j + 1]}; o[j] = __builtin_bit_cast(unsigned, b); }
      *(u32x4 *)p = o;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) p[j] = (T)v[j];
  }
}

Chunks chunks(int64_t rows, int cols, int64_t ldx) {
  const int64_t per_row = ((int64_t)cols + 31) / 32 * 4;
  return Chunks{rows * per_row, per_row, cols, ldx, cols % 32 == 0 && (ldx == cols || rows == 1)};
}
bool vector_rows(const void *x, int64_t rows, int64_t ldx, size_t es) { return ((uintptr_t)x & 15) == 0 && (rows == 1 || ldx * es % 16 == 0); }

}  // namespace

void mx_quantize(hipStream_t s, int dtype, int64_t rows, int cols, const void *x, int64_t ldx, void *codes, void *scales) {
  const Chunks g = chunks(rows, cols, ldx);
  if (g.total <= 0) return;
  const unsigned groups = (unsigned)((g.total + 255) / 256);
  if (dtype == FOCUS_F32) {
    if (vector_rows(x, rows, ldx, 4)) k_mx_quantize<float, true><<<groups, 256, 0, s>>>(g, (const float *)x, (unsigned *)codes, (unsigned char *)scales);
    else k_mx_quantize<float, false><<<groups, 256, 0, s>>>(g, (const float *)x, (unsigned *)codes, (unsigned char *)scales);
  } else {
    if (vector_rows(x, rows, ldx, 2)) k_mx_quantize<bf16_t, true><<<groups, 256, 0, s>>>(g, (const bf16_t *)x, (unsigned *)codes, (unsigned char *)scales);
    else k_mx_quantize<bf16_t, false><<<groups, 256, 0, s>>>(g, (const bf16_t *)x, (unsigned *)codes, (unsigned char *)scales);
  }
}

void mx_dequantize(hipStream_t s, int dtype, int64_t rows, int cols, focus_mx mx, void *x, int64_t ldx) {
  const Chunks g = chunks(rows, cols, ldx);
  if (g.total <= 0) return;
  const unsigned groups = (unsigned)((g.total + 255) / 256);
  const unsigned *codes = (const unsigned *)mx.codes;
  const unsigned char *scales = (const unsigned char *)mx.scales;
  if (dtype == FOCUS_F32) {
    if (vector_rows(x, rows, ldx, 4)) k_mx_dequantize<float, true><<<groups, 256, 0, s>>>(g, codes, scales, (float *)x);
    else k_mx_dequantize<float, false><<<groups, 256, 0, s>>>(g, codes, scales, (float *)x);
  } else {
    if (vector_rows(x, rows, ldx, 2)) k_mx_dequantize<bf16_t, true><<<groups, 256, 0, s>>>(g, codes, scales, (bf16_t *)x);
    else k_mx_dequantize<bf16_t, false><<<groups, 256, 0, s>>>(g, codes, scales, (bf16_t *)x);
  }
}

}  // namespace fk
