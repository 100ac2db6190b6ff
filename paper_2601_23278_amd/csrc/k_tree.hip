// Attention of drafted tokens over the paged cache.
#include "focus_branch.h"

namespace fk {

template <typename T> __device__ __forceinline__ float to_f(T v) { return (float)v; }

// One workgroup of four wavefronts per (row, query head): a wavefront takes every fourth token, all lanes on one token.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_tree_row(TreeArgs a) {
  constexpr int NE = D / 64;
  __shared__ float osh[4][D], msh[4], lsh[4];
  const int r = blockIdx.x, hq = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (r < a.cu[0] || r >= a.cu[a.n_seq]) return;
  const int H = a.g.n_kv_heads, P = a.g.page_size, h = hq / (a.n_q_heads / H);
  const int b = sequence_of(a.cu, a.n_seq, r), r0 = a.cu[b], n = min(a.cu[b + 1], a.n_rows) - r0;
  const int64_t L = max(a.lens[b], 0), total = min(L + n, (int64_t)a.g.stride * P);
  const size_t page_size = page_bytes(a.g, D, sizeof(T));
  float q[NE], o[NE], m = -INFINITY, l = 0.f;
  for (int e = 0; e < NE; ++e) {
    q[e] = to_f(((const T *)a.q)[(size_t)r * a.ldq + (size_t)hq * D + lane + 64 * e]);
    o[e] = 0.f;
  }
  for (int64_t t = wave; t < total; t += 4) {
    if (t >= L) {
      const int j = (int)(t - L);
      if (a.seen ? j >= 64 * a.seen_words || !((a.seen[(size_t)r * a.seen_words + j / 64] >> (j % 64)) & 1) : j > r - r0) continue;
    }
    const int page = page_of_token(a.g, a.g.table, a.g.stride, b, t);
    if (page < 0) continue;
    const T *kp = (const T *)(a.g.pool + (size_t)page * page_size) + ((size_t)h * P + t % P) * D;
    const T *vp = (const T *)(a.g.pool + (size_t)page * page_size) + (size_t)(H + h) * P * D + t % P;
    float s = 0.f;
    for (int e = 0; e < NE; ++e) s += q[e] * to_f(kp[lane + 64 * e]);
    for (int x = 32; x > 0; x >>= 1) s += __shfl_xor(s, x);
    s *= a.scale;
    const float mn = fmaxf(m, s), mu = mn == -INFINITY ? 0.f : mn, corr = __expf(m - mu), p = __expf(s - mu);
    l = l * corr + p;
    for (int e = 0; e < NE; ++e) o[e] = o[e] * corr + p * to_f(vp[(size_t)(lane + 64 * e) * P]);
    m = mn;
  }
  for (int e = 0; e < NE; ++e) osh[wave][lane + 64 * e] = o[e];
  if (lane == 0) { msh[wave] = m; lsh[wave] = l; }
  __syncthreads();
  if (threadIdx.x >= D) return;
  float mm = fmaxf(fmaxf(msh[0], msh[1]), fmaxf(msh[2], msh[3])), num = 0.f, den = 0.f;
  for (int w = 0; w < 4; ++w) {
    const float c = msh[w] == -INFINITY ? 0.f : __expf(msh[w] - mm);
    den += lsh[w] * c;
    num += osh[w][threadIdx.x] * c;
  }
  ((T *)a.out)[(size_t)r * a.ldo + (size_t)hq * D + threadIdx.x] = (T)(den == 0.f ? 0.f : num / den);
}

size_t tree_scratch(const TreeArgs &a) { return 0; }

void tree_attention(hipStream_t s, const TreeArgs &a) {
  const dim3 grid(a.n_rows, a.n_q_heads);
  if (a.dtype == FOCUS_F32)
    a.head_dim == 64 ? k_tree_row<float, 64><<<grid, 256, 0, s>>>(a) : k_tree_row<float, 128><<<grid, 256, 0, s>>>(a);
  else
    a.head_dim == 64 ? k_tree_row<bf16_t, 64><<<grid, 256, 0, s>>>(a) : k_tree_row<bf16_t, 128><<<grid, 256, 0, s>>>(a);
}

}  // namespace fk
