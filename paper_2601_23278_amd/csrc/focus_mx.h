// Internal declarations of the expert router and of the microscaled 4-bit (MXFP4) operators.
#pragma once

#include "focus_internal.h"

namespace fk {

// Stores the text of a failed call that has no context and returns `code`.
int fail_call(int code, const char *fmt, ...);

// ---- router -------------------------------------------------------------------------------------
struct RouteArgs {
  focus_router router;
  int dtype;                       // of the logits
  const void *logits;              // [rows, ld]
  int64_t ld;
  const float *bias;               // [E] or null
  Rows rows;
  const int32_t *row_map;          // row -> row id of the members below, null: the row itself
  const int32_t *route_override;   // [row ids, k] experts to use instead of the router's pick, or null
  int32_t *experts;                // [rows, k]
  float *weights;                  // [rows, k]
  int32_t *out_experts;            // [row ids, k] or null: the same again
  float *out_weights;
};
const char *check_router(const focus_router &r);   // what is wrong with it, or null
void route(hipStream_t s, const RouteArgs &a);

// ---- MXFP4 --------------------------------------------------------------------------------------
// A launch has at most 2^32 - 1 threads, in workgroups of 256: so many workgroups are too many.
constexpr int64_t kMaxGroups = 1 << 24;
const char *check_mx_product(int32_t m, int32_t n, int32_t k);     // what is wrong with the sizes of a product, or null
bool mx_experts_launch(int rows, int k, int n_experts, int tile_rows, int hidden, int ffn);     // the experts' grids are not too large

void mx_quantize(hipStream_t s, int dtype, int64_t rows, int cols, const void *x, int64_t ldx, void *codes, void *scales);
void mx_dequantize(hipStream_t s, int dtype, int64_t rows, int cols, focus_mx mx, void *x, int64_t ldx);

// What a product does with its sums.
enum MxEpilogue {
  MX_STORE = 0,      // out[bf16] = acc
  MX_STORE_F32 = 1,  // out[f32] = acc
  MX_ADD_F32 = 2,    // out[f32] += acc
  MX_SILU_MUL = 3    // W = [gate rows; up rows] (n = 2 F): out[bf16][m, f] = silu(gate) * up
};
// C = A W^T, A bf16 [rows, lda] or (a_scales given) MXFP4 codes [rows, k / 2]; W MXFP4 [n, k].  MX_SILU_MUL and MX_ADD_F32 with bf16 rows only.
// scratch holds the partial sums of launches that cut K (none: no such launches).
size_t mx_gemm_scratch(int rows, int n, int k, bool a_mx);
void mx_gemm(hipStream_t s, const void *a, const void *a_scales, int64_t lda, focus_mx w, int n, int k, Rows rows, int epilogue, void *out, int64_t ldo,
             Scratch scratch);

// Routed experts.  Entries (row, choice) are sorted by expert into tiles of 32 or 128 rows, multiplied expert by expert, and added up row by row.
constexpr int kMxMaxExperts = 512, kMxFewRows = 4;
struct MxExperts {
  int n_experts, hidden, ffn, k;
  focus_mx gate_up, down;
  Rows rows;
  const void *x;                  // [rows, ldx] bf16
  int64_t ldx;
  const int32_t *experts;         // [rows, k]
  const float *weights;           // [rows, k]
  int out_type;
  void *out;
  int64_t ldo;
  bool add;
  // work buffers
  int32_t *hist;                  // [mx_chunks(), E] entries of every expert in every 1024 entries
  int tile_rows;                  // 32 or 128
  int2 *tiles;                    // [mx_tile_slots()] first sorted row; expert and rows << 16
  int32_t *n_tiles;               // [1]
  int32_t *pos;                   // [rows * k] entry -> sorted row, -1: no such expert
  int32_t *arow;                  // [rows * k] sorted row -> row of x
  void *act;                      // [rows * k, ffn] bf16
  float *y;                       // [rows * k, columns of a slice]
};
int mx_tile_rows(int rows, int k, int n_experts);     // the height for so many rows: what is expected, where only the device knows
int mx_tile_slots(int rows, int k, int n_experts, int tile_rows);
int mx_chunks(int rows, int k);
size_t mx_experts_bytes(int n_experts, int hidden, int ffn, int n_rows, int k);
void lay_mx_experts(MxExperts &a, void *workspace);
void mx_group(hipStream_t s, const MxExperts &a);     // entries sorted by expert, tiles
void mx_up(hipStream_t s, const MxExperts &a);        // act
void mx_down(hipStream_t s, const MxExperts &a);      // second product and weighted sum

}  // namespace fk
