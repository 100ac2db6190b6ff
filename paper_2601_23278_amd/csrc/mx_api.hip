// C entries of the expert router and of the MXFP4 operators that need no context: argument checks and launches.
#include <algorithm>

#include "focus_mx.h"

using fk::fail_call;

namespace {

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// What a launch that went wrong left behind, as this call's error.
int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FOCUS_OK : fail_call(FOCUS_EHIP, "launch: %s", hipGetErrorString(e));
}

const char *check_product(int32_t m, int32_t n, int32_t k, int32_t a_type) {
  if (a_type != FOCUS_BF16 && a_type != FOCUS_MX4) return "a_type must be FOCUS_BF16 or FOCUS_MX4";
  return fk::check_mx_product(m, n, k);
}

const char *check_experts(int32_t n_experts, int32_t hidden, int32_t ffn, int32_t n_rows, int32_t k) {
  if (n_experts < 1 || n_experts > fk::kMxMaxExperts) return "n_experts must be in 1..512";
  if (hidden < 32 || hidden % 32 || ffn < 32 || ffn % 32) return "hidden and ffn must be positive multiples of 32";
  if (hidden > (1 << 20) || ffn > (1 << 20) || (int64_t)hidden * ffn >= (1ll << 31)) return "hidden and ffn too large";
  if (n_rows < 0 || k < 1 || k > 32 || (int64_t)n_rows * k >= (1 << 24)) return "n_rows must not be negative, k in 1..32 and n_rows * k below 2^24";
  if (!fk::mx_experts_launch(n_rows, k, n_experts, fk::mx_tile_rows(n_rows, k, n_experts), hidden, ffn)) return "hidden, ffn and n_rows too large";
  return nullptr;
}

}  // namespace

const char *fk::check_mx_product(int32_t m, int32_t n, int32_t k) {
  if (m < 0 || n < 0 || k < 0 || k % 32) return "m, n and k must not be negative and k a multiple of 32";
  if (k > (1 << 22)) return "k must be at most 2^22";
  if ((int64_t)n * (k / 2) >= (1ll << 31) || ((int64_t)m + 127) / 128 * (((int64_t)n + 127) / 128) > kMaxGroups - 8) return "m, n and k too large";   // rounded up to the eight XCDs
  return nullptr;
}

bool fk::mx_experts_launch(int rows, int k, int n_experts, int tile_rows, int hidden, int ffn) {      // a workgroup per 128 columns and tile of rows
  return (int64_t)mx_tile_slots(rows, k, n_experts, tile_rows) * ((std::max(hidden, 2 * ffn) + 127) / 128) < kMaxGroups;
}

extern "C" {

int focus_route(const focus_router *router, void *hip_stream, int32_t n_rows, int32_t dtype, const void *logits, int64_t ld, const float *bias,
                int32_t *experts, float *weights) {
  if (!router) return fail_call(FOCUS_EINVAL, "null router");
  if (const char *e = fk::check_router(*router)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (n_rows < 0 || n_rows > 4 * (fk::kMaxGroups - 1)) return fail_call(FOCUS_EINVAL, "n_rows must be in 0..2^26 - 4");         // four rows a workgroup
  if (dtype != FOCUS_F32 && dtype != FOCUS_BF16) return fail_call(FOCUS_EINVAL, "dtype must be FOCUS_F32 or FOCUS_BF16");
  if (ld < router->n_experts) return fail_call(FOCUS_EINVAL, "ld is less than n_experts");
  if (n_rows == 0) return FOCUS_OK;
  if (!logits || !experts || !weights) return fail_call(FOCUS_EINVAL, "null logits, experts or weights");
  if (!aligned(logits, dtype == FOCUS_F32 ? 4 : 2) || !aligned(bias, 4) || !aligned(experts, 4) || !aligned(weights, 4)) return fail_call(FOCUS_EINVAL, "a pointer is not aligned to its elements");
  fk::RouteArgs a{};
  a.router = *router; a.dtype = dtype; a.logits = logits; a.ld = ld; a.bias = bias; a.rows = fk::Rows{n_rows, nullptr}; a.experts = experts; a.weights = weights;
  fk::route((hipStream_t)hip_stream, a);
  return launched();
}

static int check_conversion(int32_t dtype, int64_t rows, int32_t cols, const void *x, int64_t ldx, const void *codes, const void *scales) {
  if (dtype != FOCUS_F32 && dtype != FOCUS_BF16) return fail_call(FOCUS_EINVAL, "dtype must be FOCUS_F32 or FOCUS_BF16");
  if (rows < 0 || cols < 0) return fail_call(FOCUS_EINVAL, "rows and cols must not be negative");
  if (ldx < cols) return fail_call(FOCUS_EINVAL, "ldx is less than cols");
  // 64 blocks of 32 a workgroup
  if (rows >= (1ll << 30) || rows * (((int64_t)cols + 31) / 32) > 64 * (fk::kMaxGroups - 1)) return fail_call(FOCUS_EINVAL, "rows and cols too large");
  if (rows == 0 || cols == 0) return FOCUS_OK;
  if (!x || !codes || !scales) return fail_call(FOCUS_EINVAL, "null x, codes or scales");
  if (!aligned(codes, 16)) return fail_call(FOCUS_EINVAL, "codes must be 16-byte aligned");
  if (!aligned(x, dtype == FOCUS_F32 ? 4 : 2)) return fail_call(FOCUS_EINVAL, "x is not aligned to its elements");
  return FOCUS_OK;
}

int focus_mx_quantize(void *hip_stream, int32_t dtype, int64_t rows, int32_t cols, const void *x, int64_t ldx, void *codes, void *scales) {
  if (int rc = check_conversion(dtype, rows, cols, x, ldx, codes, scales)) return rc;
  if (rows == 0 || cols == 0) return FOCUS_OK;
  fk::mx_quantize((hipStream_t)hip_stream, dtype, rows, cols, x, ldx, codes, scales);
  return launched();
}

int focus_mx_dequantize(void *hip_stream, int32_t dtype, int64_t rows, int32_t cols, const focus_mx *mx, void *x, int64_t ldx) {
  if (!mx) return fail_call(FOCUS_EINVAL, "null mx");
  if (int rc = check_conversion(dtype, rows, cols, x, ldx, mx->codes, mx->scales)) return rc;
  if (rows == 0 || cols == 0) return FOCUS_OK;
  fk::mx_dequantize((hipStream_t)hip_stream, dtype, rows, cols, *mx, x, ldx);
  return launched();
}

int focus_mx_gemm_bytes(int32_t m, int32_t n, int32_t k, int32_t a_type, size_t *bytes) {
  if (!bytes) return fail_call(FOCUS_EINVAL, "null bytes");
  if (const char *e = check_product(m, n, k, a_type)) return fail_call(FOCUS_EINVAL, "%s", e);
  *bytes = m > 0 && n > 0 ? fk::mx_gemm_scratch(m, n, k, a_type == FOCUS_MX4) : 0;
  return FOCUS_OK;
}

int focus_mx_gemm(void *hip_stream, int32_t m, int32_t n, int32_t k, int32_t a_type, const void *a, const void *a_scales, int64_t lda, const focus_mx *w,
                  int32_t c_type, void *c, int64_t ldc, void *workspace, size_t workspace_bytes) {
  if (const char *e = check_product(m, n, k, a_type)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (c_type != FOCUS_F32 && c_type != FOCUS_BF16) return fail_call(FOCUS_EINVAL, "c_type must be FOCUS_F32 or FOCUS_BF16");
  if (!w) return fail_call(FOCUS_EINVAL, "null w");
  if (ldc < n) return fail_call(FOCUS_EINVAL, "ldc is less than n");
  if (a_type == FOCUS_BF16 && (lda < k || lda % 8 || lda > (1 << 22))) return fail_call(FOCUS_EINVAL, "lda must be a multiple of 8, at least k and at most 2^22");
  if (m == 0 || n == 0) return FOCUS_OK;
  if (!c || (k > 0 && (!a || !w->codes || !w->scales))) return fail_call(FOCUS_EINVAL, "null operand");
  if (k > 0 && ((a_type == FOCUS_MX4) != (a_scales != nullptr))) return fail_call(FOCUS_EINVAL, "a_scales belong to FOCUS_MX4 rows");
  if (!aligned(a, 16) || !aligned(w->codes, 16) || !aligned(workspace, 16)) return fail_call(FOCUS_EINVAL, "a, the codes and the workspace must be 16-byte aligned");
  if (!aligned(c, c_type == FOCUS_F32 ? 4 : 2)) return fail_call(FOCUS_EINVAL, "c is not aligned to its elements");
  fk::mx_gemm((hipStream_t)hip_stream, a, a_scales, lda, *w, n, k, fk::Rows{m, nullptr}, c_type == FOCUS_F32 ? fk::MX_STORE_F32 : fk::MX_STORE, c, ldc,
              fk::Scratch{workspace, workspace ? workspace_bytes : 0});
  return launched();
}

int focus_mx_experts_bytes(int32_t n_experts, int32_t hidden, int32_t ffn, int32_t n_rows, int32_t k, size_t *bytes) {
  if (!bytes) return fail_call(FOCUS_EINVAL, "null bytes");
  if (const char *e = check_experts(n_experts, hidden, ffn, n_rows, k)) return fail_call(FOCUS_EINVAL, "%s", e);
  *bytes = fk::mx_experts_bytes(n_experts, hidden, ffn, n_rows, k);
  return FOCUS_OK;
}

int focus_mx_experts(void *hip_stream, int32_t n_experts, int32_t hidden, int32_t ffn, const focus_mx *gate_up, const focus_mx *down, int32_t n_rows, int32_t k,
                     const void *x, int64_t ldx, const int32_t *experts, const float *weights, int32_t out_type, void *out, int64_t ldo, int32_t add,
                     void *workspace, size_t workspace_bytes) {
  if (const char *e = check_experts(n_experts, hidden, ffn, n_rows, k)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (out_type != FOCUS_F32 && out_type != FOCUS_BF16) return fail_call(FOCUS_EINVAL, "out_type must be FOCUS_F32 or FOCUS_BF16");
  if ((add != 0 && add != 1) || (add && out_type != FOCUS_F32)) return fail_call(FOCUS_EINVAL, "add must be 0 or 1, and 0 with FOCUS_BF16");
  if (ldx < hidden || ldx % 8 || ldo < hidden) return fail_call(FOCUS_EINVAL, "ldx must be a multiple of 8, ldx and ldo at least hidden");
  if (n_rows > 0 && ldx >= (1ll << 30) / n_rows) return fail_call(FOCUS_EINVAL, "n_rows * ldx must be below 2^30");
  if (n_rows == 0) return FOCUS_OK;
  if (!gate_up || !down || !gate_up->codes || !gate_up->scales || !down->codes || !down->scales || !x || !experts || !weights || !out || !workspace)
    return fail_call(FOCUS_EINVAL, "null operand");
  if (!aligned(gate_up->codes, 16) || !aligned(down->codes, 16) || !aligned(x, 16)) return fail_call(FOCUS_EINVAL, "x and the codes must be 16-byte aligned");
  if (!aligned(workspace, 256) || !aligned(experts, 4) || !aligned(weights, 4) || !aligned(out, out_type == FOCUS_F32 ? 4 : 2))
    return fail_call(FOCUS_EINVAL, "workspace must be 256-byte aligned, the others to their elements");
  if (workspace_bytes < fk::mx_experts_bytes(n_experts, hidden, ffn, n_rows, k)) return fail_call(FOCUS_ENOMEM, "the workspace is too small");
  fk::MxExperts a{};
  a.n_experts = n_experts; a.hidden = hidden; a.ffn = ffn; a.k = k; a.gate_up = *gate_up; a.down = *down; a.rows = fk::Rows{n_rows, nullptr};
  a.x = x; a.ldx = ldx; a.experts = experts; a.weights = weights; a.out_type = out_type; a.out = out; a.ldo = ldo; a.add = add != 0;
  fk::lay_mx_experts(a, workspace);
  fk::mx_group((hipStream_t)hip_stream, a);
  fk::mx_up((hipStream_t)hip_stream, a);
  fk::mx_down((hipStream_t)hip_stream, a);
  return launched();
}

}  // extern "C"
