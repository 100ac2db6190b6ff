// Internal declarations of the operators for generation that branches over the paged cache (tree attention, page bookkeeping, beam selection).
#pragma once

#include "focus_mx.h"

namespace fk {

// A page table and the pool it points into, as kernels see them.
struct Paged {
  char *pool;                 // of one layer, or of the first one
  int n_pages, page_size, n_kv_heads, n_layers;
  const int32_t *table;
  int stride;
};

// Bytes of a page; es = bytes of an element.
__host__ __device__ __forceinline__ size_t page_bytes(const Paged &g, int head_dim, int es) { return (size_t)2 * g.n_kv_heads * g.page_size * head_dim * es; }
// Where token t of row b lies; page -1: nowhere.  Tokens are below 2^32 (a length and a position, 31 bits each).
struct Place {
  int page, at;
};
__device__ __forceinline__ Place place_of(const Paged &g, const int32_t *table, int stride, int b, int64_t t) {
  const unsigned i = (unsigned)t / (unsigned)g.page_size;
  const int p = t >= 0 && i < (unsigned)stride ? table[(size_t)b * stride + i] : -1;
  return Place{p < g.n_pages ? p : -1, (int)((unsigned)t - i * (unsigned)g.page_size)};
}
// The last b with cu[b] <= r among 0..n - 1 (n >= 1).  The caller checks that r < cu[b + 1].
__device__ __forceinline__ int sequence_of(const int32_t *cu, int n, int r) {
  int lo = 0, hi = n;                       // cu[lo] <= r (if any is), cu[hi] > r or hi == n
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (cu[mid] <= r) lo = mid; else hi = mid;
  }
  return lo;
}

struct AppendArgs {
  int dtype, head_dim;
  Paged g;
  int n_seq, n_rows;
  const int32_t *cu, *lens;
  const void *k, *v;
  int64_t ldk, ldv;
};
void kv_append(hipStream_t s, const AppendArgs &a);

struct TreeArgs {
  int dtype, head_dim;
  Paged g;
  int n_seq, n_rows, n_q_heads, seen_words;
  int max_rows, max_len;            // what the host knows, 0: nothing
  const int32_t *cu, *lens;
  const uint64_t *seen;
  float scale;
  const void *q;
  void *out;
  int64_t ldq, ldo;
  Scratch scratch;
};
size_t tree_scratch(const TreeArgs &a);
void tree_attention(hipStream_t s, const TreeArgs &a);

struct CompactArgs {
  int dtype, head_dim;
  Paged g;                          // the tables that tokens are read by
  int n_seq, n_keep;
  const int32_t *start, *cu, *keep;
  const int32_t *to_table;
  int to_stride;
};
void kv_compact(hipStream_t s, const CompactArgs &a);

struct ForkArgs {
  int dtype, head_dim;
  Paged g;
  int n_old, n_new;
  const int32_t *parents, *lens;
  int32_t *new_lens, *new_table, *refs, *lacking;
  int32_t *work;                    // [fork_ints(n_new)]
};
inline size_t fork_ints(int n_new) { return 4 * (size_t)n_new + 4; }
void kv_fork(hipStream_t s, const ForkArgs &a);

struct ReserveArgs {
  int n_seq, page_size, n_pages, room, stride;
  const int32_t *lens;
  int32_t *table, *refs, *lacking;
  int32_t *work;                    // [reserve_ints(n_seq)]
};
inline size_t reserve_ints(int n_seq) { return 3 * (size_t)n_seq + 4; }
void kv_reserve(hipStream_t s, const ReserveArgs &a);

constexpr int kMaxBeams = 64, kMaxPicks = 64;
struct BeamArgs {
  int n_seq, n_beams, vocab, k, dtype;
  const void *logits;
  int64_t ld;
  const float *scores;
  const uint8_t *done;
  int end_token;
  int32_t *rows, *tokens;
  float *new_scores;
  void *work;                       // beam_scratch() bytes
};
int64_t beam_groups(int n_seq, int n_beams, int vocab, int k);     // workgroups of the larger launch
size_t beam_scratch(int n_seq, int n_beams, int vocab, int k);
void beam_select(hipStream_t s, const BeamArgs &a);

}  // namespace fk
