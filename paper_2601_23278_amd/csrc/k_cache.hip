// The paged cache of sequences that branch: rows of K/V into pages, tokens that stay moved together, pages shared, copied, given out and given back.
//
// A page holds K [H_kv][P][D], then V transposed [H_kv][D][P]: a token is a row of 2 D bytes (bf16) in K and a column in V.  All of these are bound by
// the bytes they move (nothing is computed) or, for a request's few tokens, by a chain of dependent loads: row -> sequence -> page -> data.
#include "focus_branch.h"

namespace fk {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
template <int ES> struct Word;
template <> struct Word<2> { typedef uint16_t type; };
template <> struct Word<4> { typedef uint32_t type; };

// ---------------------------------------------------------------------------------------------
// Append.  A workgroup takes 64 rows of one kv head (in row order, whatever their sequences).  K rows are copied in 16-byte pieces; V goes through LDS, so that
// the lanes of a wavefront are 64 rows and a store of one d writes neighbouring tokens of a page.
template <int ES, int D>
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
  typedef typename Word<ES>::type T;
  constexpr int PIECES = D * ES / 16, PER = 16 / ES;
  __shared__ int page_s[64], place_s[64];
  __shared__ T vs[64][D + 16 / ES / 2];
  const int r0 = blockIdx.x * 64, h = blockIdx.y, tid = threadIdx.x, P = a.g.page_size;
  if (tid < 64) {
    const int r = r0 + tid;
    Place at{-1, 0};
    if (r < a.n_rows && r >= a.cu[0] && r < a.cu[a.n_seq]) {
      const int b = sequence_of(a.cu, a.n_seq, r);
      const int64_t t = (int64_t)max(a.lens[b], 0) + r - a.cu[b];
      at = place_of(a.g, a.g.table, a.g.stride, b, t);
    }
    page_s[tid] = at.page;
    place_s[tid] = at.at;
  }
  __syncthreads();
  const T *k = (const T *)a.k + (size_t)h * D, *v = (const T *)a.v + (size_t)h * D;
  const size_t page_size = page_bytes(a.g, D, ES);
  const bool wide = ((uintptr_t)k % 16 == 0) && ((uintptr_t)v % 16 == 0) && (a.ldk * ES) % 16 == 0 && (a.ldv * ES) % 16 == 0;
  for (int i = tid; i < 64 * PIECES; i += 256) {
    const int row = i / PIECES, c = i % PIECES, page = page_s[row];
    if (page < 0) continue;
    T *to = (T *)(a.g.pool + (size_t)page * page_size) + ((size_t)h * P + place_s[row]) * D + c * PER;
    const T *kr = k + (size_t)(r0 + row) * a.ldk + c * PER, *vr = v + (size_t)(r0 + row) * a.ldv + c * PER;
    if (wide) {
      const u32x4 kk = *(const u32x4 *)kr, vv = *(const u32x4 *)vr;
      *(u32x4 *)to = kk;
#pragma unroll
      for (int e = 0; e < PER; ++e) vs[row][c * PER + e] = ((const T *)&vv)[e];
    } else {
      for (int e = 0; e < PER; ++e) {
        to[e] = kr[e];
        vs[row][c * PER + e] = vr[e];
      }
    }
  }
  __syncthreads();
  const int row = tid & 63, page = page_s[row];
  if (page < 0) return;
  T *to = (T *)(a.g.pool + (size_t)page * page_size) + (size_t)(a.g.n_kv_heads + h) * P * D + place_s[row];
  for (int d = tid >> 6; d < D; d += 4) to[(size_t)d * P] = vs[row][d];
}

void kv_append(hipStream_t s, const AppendArgs &a) {
  const dim3 grid((a.n_rows + 63) / 64, a.g.n_kv_heads);
  if (a.dtype == FOCUS_F32)
    a.head_dim == 64 ? k_append<4, 64><<<grid, 256, 0, s>>>(a) : k_append<4, 128><<<grid, 256, 0, s>>>(a);
  else
    a.head_dim == 64 ? k_append<2, 64><<<grid, 256, 0, s>>>(a) : k_append<2, 128><<<grid, 256, 0, s>>>(a);
}

// ---------------------------------------------------------------------------------------------
// Compaction.  A workgroup takes one (sequence, head, layer), or a slice of its columns where those are few, and moves tokens in ascending order, 64 at a time.
// In place that is safe: place i is read from place keep[i] >= i, so nothing that was written is read later; and every column of K (16 bytes) and every row of
// V^T belongs to one wavefront, which loads all of a batch before it stores any of it.  So wavefronts do not wait for each other's data, only for the list of
// where the next 256 tokens move: `keep` of them is asked for ahead of the last ones' moves, their pages are looked up behind them.  Batches begin at every 64th token of what is written: a store to V^T fills a line.
// Rows of V^T that a batch's tokens come from are read in whole 16-byte pieces into LDS and picked from there, 16 bytes of neighbouring tokens a store, as long as
// they span at most 256 tokens: single values, 64 lanes from three or four lines, took 342 us for a third of 8 x 8000 tokens (4 layers), this takes 263.
template <int ES, int D, int SLICES>
__global__ __launch_bounds__(256) void k_compact(CompactArgs a) {
  typedef typename Word<ES>::type T;
  // Columns of K of the workgroup, and of a wavefront that has any: at least four, so that its 16 bytes a lane lie side by side.  Rows of V^T of the workgroup.
  constexpr int ALL_COLS = D * ES / 16 / SLICES, COLS = ALL_COLS / 4 < 4 ? 4 : ALL_COLS / 4, ROWS = D / SLICES;
  constexpr int TOKENS = 64 / COLS, NK = COLS, NV = ROWS / 4 < 8 ? ROWS / 4 : 8;
  constexpr int RW = ROWS / 4, RG = RW < 8 ? RW : 8, SPAN = 256;           // rows of V^T of a wavefront, and of them at a time; tokens held of each
  __shared__ int4 move_s[2][256];                      // pages and places, from and to
  __shared__ int token_s[2][256];                      // tokens that move, counted from the last 8th one up to `start`; -1: none
  __shared__ __attribute__((aligned(16))) T stage_s[4][RG][SPAN + 16 / ES];      // rows four banks apart
  const int H = a.g.n_kv_heads, b = blockIdx.x / H, h = blockIdx.x % H, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, P = a.g.page_size;
  const int c0 = min(max(a.cu[b], 0), a.n_keep), n = min(a.cu[b + 1], a.n_keep) - c0;
  if (n <= 0) return;
  const int64_t start = max(a.start[b], 0), base = start & ~(int64_t)63;
  const int skip = (int)(start - base), end = skip + n;      // places base + j, skip <= j < end, are written
  const size_t page_size = page_bytes(a.g, D, ES);
  char *const pool = a.g.pool + (size_t)blockIdx.y * a.g.n_pages * page_size;
  const size_t k_head = (size_t)h * P * D * ES + (blockIdx.z * ALL_COLS + wave * COLS) * 16, v_head = (size_t)(H + h) * P * D * ES + (size_t)blockIdx.z * ROWS * P * ES;
  auto kept = [&](int j) { return j >= skip && j < end ? a.keep[c0 + j - skip] : -1; };
  const int past = (int)(start & 7);
  const int64_t start8 = start - past;
  auto where = [&](int j, int keep) {
    if (j < skip || j >= end) return int4{-1, 0, -1, 0};
    const Place from = place_of(a.g, a.g.table, a.g.stride, b, keep < 0 ? -1 : start + keep), to = place_of(a.g, a.to_table, a.to_stride, b, base + j);
    return int4{from.page, from.at, from.page < 0 ? -1 : to.page, to.at};
  };
  // A few tokens in all are told apart by few lanes of V's loads; else a lane is a token.
  const bool few = end - skip <= 32;
  const int bits = !few ? 6 : n > 16 ? 5 : n > 8 ? 4 : n > 4 ? 3 : n > 2 ? 2 : n - 1, by = 256 >> bits;
  const int keep_0 = kept(tid);
  move_s[0][tid] = where(tid, keep_0);
  token_s[0][tid] = move_s[0][tid].z >= 0 ? keep_0 + past : -1;
  __syncthreads();
  for (int j0 = 0, buf = 0; j0 < end; j0 += 256, buf ^= 1) {
    const int next = kept(j0 + 256 + tid);
    const int last = min(end - j0, 256), begin = max(skip - j0, 0);
    // with few tokens one batch from the first token on, across the 64
    for (int s0 = few ? begin : 0; s0 < last; s0 += 64) {
      const int lo = max(begin, s0), hi = min(last, s0 + 64);
      int4 km[NK];
      u32x4 kk[NK];
#pragma unroll
      for (int x = 0; x < NK; ++x) {
        const int t = lo + x * TOKENS + lane / COLS;
        km[x] = t < hi && wave * COLS < ALL_COLS ? move_s[buf][t] : int4{-1, 0, -1, 0};
        if (km[x].z >= 0) kk[x] = *(const u32x4 *)(pool + (size_t)km[x].x * page_size + k_head + (size_t)km[x].y * D * ES + lane % COLS * 16);
      }
      bool staged = false;
      if (!few) {
        // chunk: the 8 tokens that the first of the batch is among; all others have to lie in the SPAN tokens from there
        const int mine = s0 + lane >= lo && s0 + lane < hi ? token_s[buf][s0 + lane] : -1;
        const uint64_t some = __ballot(mine >= 0);
        const int chunk = some ? __builtin_amdgcn_readlane(mine, __builtin_ctzll(some)) >> 3 : 0;
        staged = __ballot(mine >= 0 && (mine < chunk * 8 || mine >= chunk * 8 + SPAN)) == 0;
        if (staged && some) {
          const int last = __builtin_amdgcn_readlane(mine, 63 - __builtin_clzll(some)) >> 3;      // ascending: the last chunk too
          const Place from = place_of(a.g, a.g.table, a.g.stride, b, start8 + (int64_t)(chunk + (lane & 31)) * 8);
          const bool reads = from.page >= 0 && chunk + (lane & 31) <= last;
          const T *const src = (const T *)(pool + (size_t)max(from.page, 0) * page_size + v_head) + from.at;
          const int grp = lane & 7, r_out = lane >> 3;                 // a lane stores 8 neighbouring tokens of one row
          int pick[8];
          bool full = true;
          int4 to_8 = {-1, 0, -1, 0};
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int t = s0 + grp * 8 + e;
            const int tok = t >= lo && t < hi ? token_s[buf][t] : -1;
            pick[e] = tok < 0 ? -1 : tok - chunk * 8;
            full &= tok >= 0;
            if (tok >= 0) to_8 = move_s[buf][t];
          }
          // the group's 8 tokens begin at a multiple of 8 and lie in one page
          T *const out = (T *)(pool + (size_t)max(to_8.z, 0) * page_size + v_head) + (to_8.w & ~7);
          for (int r0 = 0; r0 < RW; r0 += RG) {
#pragma unroll
            for (int x = 0; x < RG / 2; ++x) {
              const int r = x * 2 + (lane >> 5);
              if (reads) {
                const u32x4 *const from_row = (const u32x4 *)(src + (size_t)(wave * RW + r0 + r) * P);
#pragma unroll
                for (int y = 0; y < ES / 2; ++y) *(u32x4 *)&stage_s[wave][r][(lane & 31) * 8 + y * (16 / ES)] = from_row[y];
              }
            }
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
            if (r_out < RG && to_8.z >= 0) {
              T v[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e] = stage_s[wave][r_out][max(pick[e], 0)];
              T *const row = out + (size_t)(wave * RW + r0 + r_out) * P;
              if (full) {
#pragma unroll
                for (int y = 0; y < ES / 2; ++y) ((u32x4 *)row)[y] = *(const u32x4 *)&v[y * (16 / ES)];
              } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  if (pick[e] >= 0) row[e] = v[e];
              }
            }
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");
          }
        }
      }
      if (!staged) {
        // Few tokens in all are told apart by few lanes; else a lane is a token, and the rows are those of the other form.
        const int vt = s0 + (tid & ((1 << bits) - 1)), vd = few ? tid >> bits : wave * RW, step = few ? by : 1, v_end = few ? ROWS : wave * RW + RW;
        const int4 vm = vt >= lo && vt < hi ? move_s[buf][vt] : int4{-1, 0, -1, 0};
        const T *const vf = (const T *)(pool + (size_t)max(vm.x, 0) * page_size + v_head) + vm.y;
        T *const vto = (T *)(pool + (size_t)max(vm.z, 0) * page_size + v_head) + vm.w;
        for (int d0 = vd; d0 < v_end; d0 += step * NV) {
          T vv[NV];
#pragma unroll
          for (int x = 0; x < NV; ++x)
            if (vm.z >= 0 && d0 + step * x < v_end) vv[x] = vf[(size_t)(d0 + step * x) * P];
#pragma unroll
          for (int x = 0; x < NV; ++x)
            if (vm.z >= 0 && d0 + step * x < v_end) vto[(size_t)(d0 + step * x) * P] = vv[x];
        }
      }
#pragma unroll
      for (int x = 0; x < NK; ++x)
        if (km[x].z >= 0) *(u32x4 *)(pool + (size_t)km[x].z * page_size + k_head + (size_t)km[x].w * D * ES + lane % COLS * 16) = kk[x];
    }
    if (j0 + 256 < end) {
      const int4 then = where(j0 + 256 + tid, next);
      move_s[buf ^ 1][tid] = then;
      token_s[buf ^ 1][tid] = then.z >= 0 ? next + past : -1;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the list is there; stores need not be
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
  }
}

template <int ES, int D>
void compact_of(hipStream_t s, const CompactArgs &a) {
  constexpr int SLICES = D * ES / 16 / 4 < 4 ? D * ES / 16 / 4 : 4;
  const int groups = a.n_seq * a.g.n_kv_heads;
  if ((int64_t)groups * a.g.n_layers <= 1024)
    k_compact<ES, D, SLICES><<<dim3(groups, a.g.n_layers, SLICES), 256, 0, s>>>(a);
  else
    k_compact<ES, D, 1><<<dim3(groups, a.g.n_layers), 256, 0, s>>>(a);
}
void kv_compact(hipStream_t s, const CompactArgs &a) {
  if (a.dtype == FOCUS_F32)
    a.head_dim == 64 ? compact_of<4, 64>(s, a) : compact_of<4, 128>(s, a);
  else
    a.head_dim == 64 ? compact_of<2, 64>(s, a) : compact_of<2, 128>(s, a);
}

// ---------------------------------------------------------------------------------------------
// Page bookkeeping.

// Entries of a row up to the first negative one; the whole workgroup.
__device__ int held_pages(const int32_t *row, int stride) {
  __shared__ int first;
  for (int j0 = 0; j0 < stride; j0 += blockDim.x) {
    if (threadIdx.x == 0) first = stride;
    __syncthreads();
    const int j = j0 + threadIdx.x;
    if (j < stride && row[j] < 0) atomicMin(&first, j);
    __syncthreads();
    const int f = first;
    __syncthreads();
    if (f < stride) return f;
  }
  return stride;
}

// Work buffers of a fork: per new row whether it wants a page, the page it copies from, the page it got (-1: none), and the tokens to copy.
struct ForkWork {
  int32_t *start, *from, *to, *tokens;
};
__host__ __device__ inline ForkWork fork_work(const ForkArgs &a) {
  return ForkWork{a.work, a.work + a.n_new + 1, a.work + 2 * (size_t)a.n_new + 1, a.work + 3 * (size_t)a.n_new + 1};
}

// Workgroups 0 .. n_old - 1: what an old row held changes by its children.  The others: the entries of a new row.  The counts are whole numbers, so the order of
// the atomics does not show.
__global__ __launch_bounds__(256) void k_fork_rows(ForkArgs a) {
  __shared__ int count;
  const int tid = threadIdx.x, P = a.g.page_size, stride = a.g.stride;
  const bool old = (int)blockIdx.x < a.n_old;
  const int i = old ? blockIdx.x : blockIdx.x - a.n_old;
  const int p = old ? i : a.parents[i];
  const bool valid = p >= 0 && p < a.n_old;
  if (tid == 0) count = 0;
  __syncthreads();
  int mine = 0;                                        // children of an old row; of a new one, those of its parent before it
  for (int j = tid; j < (old ? a.n_new : i); j += 256) mine += a.parents[j] == p;
  if (mine) atomicAdd(&count, mine);
  __syncthreads();
  const int32_t *row = a.g.table + (size_t)(valid ? p : 0) * stride;
  const int held = valid ? held_pages(row, stride) : 0;
  const int64_t room = (int64_t)held * P;
  const int len = valid ? (int)min((int64_t)max(a.lens[p], 0), room) : 0;
  const int whole = len / P, left = len % P;
  if (old) {
    for (int j = tid; j < held; j += 256) {
      const int change = j < whole ? count - 1 : count > 0 ? 0 : -1, page = row[j];
      if (change && page < a.g.n_pages) atomicAdd(&a.refs[page], change);
    }
    return;
  }
  const int keeps = count == 0 ? held : whole;         // the first child takes everything
  int32_t *to = a.new_table + (size_t)i * stride;
  for (int j = tid; j < stride; j += 256) to[j] = j < keeps ? row[j] : -1;
  if (tid == 0) {
    const ForkWork w = fork_work(a);
    const bool wants = valid && count > 0 && left > 0;
    a.new_lens[i] = len;
    w.start[i] = wants;
    w.from[i] = wants ? row[whole] : -1;
    w.tokens[i] = left;
    w.to[i] = -1;
  }
}

// Sum of v over the threads before this one; *all = the sum of all.  `part` holds one value per wavefront.
__device__ __forceinline__ int sum_before(int v, int *part, int *all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = blockDim.x >> 6;
  int x = v;
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == 63) part[wave] = x;
  __syncthreads();
  int y = lane < n ? part[lane] : 0, before = 0;       // every wavefront sums up the others
#pragma unroll 1
  for (int w = 0; w < n; ++w) {
    const int s = __builtin_amdgcn_readlane(y, w);
    before += w < wave ? s : 0;
    *all = w == 0 ? s : *all + s;
  }
  __syncthreads();
  return before + x - v;
}

// One workgroup.  start[i]: pages that row i wants; becomes the number of pages wanted by the rows before it, and tell(i, wants, before) is called.  Returns the sum.
template <typename F>
__device__ int order_wants(int32_t *start, int n, int *part, F tell) {
  int total = 0;
  for (int i0 = 0; i0 < n; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x, v = i < n ? start[i] : 0;
    int all;
    const int before = total + sum_before(v, part, &all);
    if (i < n) {
      start[i] = before;
      tell(i, v, before);
    }
    total += all;
  }
  if (threadIdx.x == 0) start[n] = total;
  __syncthreads();
  return total;
}

// One workgroup: hands the lowest free pages out, give(rank, page) for page number `rank` of those wanted.  Returns how many there were.
template <typename F>
__device__ int hand_out(int32_t *refs, int n_pages, int wanted, int *part, F give) {
  int found = 0;
  for (int p0 = 0; p0 < n_pages && found < wanted; p0 += 4 * blockDim.x) {
    const int p = p0 + 4 * threadIdx.x;
    int free[4], mine = 0, all;
#pragma unroll
    for (int e = 0; e < 4; ++e) free[e] = refs[min(p + e, n_pages - 1)];
#pragma unroll
    for (int e = 0; e < 4; ++e) mine += free[e] = p + e < n_pages && free[e] == 0;
    int rank = found + sum_before(mine, part, &all);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (free[e]) {
        if (rank < wanted) {
          refs[p + e] = 1;
          give(rank, p + e);
        }
        ++rank;
      }
    found += all;
  }
  __syncthreads();
  return min(found, wanted);
}

// Rows that want a page, in their order; up to kWantsInLds of them are told to the page that they get without a search in memory.
constexpr int kWantsInLds = 4096;
__global__ __launch_bounds__(1024) void k_fork_pages(ForkArgs a) {
  __shared__ int part[16];
  __shared__ int who[kWantsInLds];
  const ForkWork w = fork_work(a);
  const int wanted = order_wants(w.start, a.n_new, part, [&](int i, int v, int before) {
    if (v && before < kWantsInLds) who[before] = i;
    a.lacking[i] = 0;
  });
  const int got = hand_out(a.refs, a.g.n_pages, wanted, part, [&](int rank, int page) {
    const int i = rank < kWantsInLds ? who[rank] : sequence_of(w.start, a.n_new, rank);
    w.to[i] = page;
    a.new_table[(size_t)i * a.g.stride + a.new_lens[i] / a.g.page_size] = page;
  });
  for (int rank = got + threadIdx.x; rank < wanted; rank += blockDim.x) {      // no page was left
    const int i = rank < kWantsInLds ? who[rank] : sequence_of(w.start, a.n_new, rank);
    a.lacking[i] = 1;
    a.new_lens[i] -= w.tokens[i];
  }
}

// The tokens of a page that has begun, into a page of the row's own: one head of one layer a workgroup.
template <int ES>
__global__ __launch_bounds__(256) void k_fork_copy(ForkArgs a) {
  typedef typename Word<ES>::type T;
  constexpr int PER = 16 / ES;
  const ForkWork w = fork_work(a);
  const int H = a.g.n_kv_heads, i = blockIdx.x / H, h = blockIdx.x % H, P = a.g.page_size, D = a.head_dim;
  const int from = w.from[i], to = w.to[i], n = w.tokens[i];
  if (to < 0 || from < 0 || from >= a.g.n_pages) return;
  const size_t page_size = page_bytes(a.g, D, ES);
  char *const pool = a.g.pool + (size_t)blockIdx.y * a.g.n_pages * page_size;
  const char *src = pool + (size_t)from * page_size;
  char *dst = pool + (size_t)to * page_size;
  const size_t k0 = (size_t)h * P * D * ES, v0 = (size_t)(H + h) * P * D * ES;
  const int row = D * ES / 16, pieces = (n + PER - 1) / PER, k_pieces = n * row, all = k_pieces + D * pieces;      // 16 bytes each
  auto offset = [&](int j) {                           // of piece j: K's rows, then the begun pieces of V^T's
    if (j < k_pieces) return k0 + (size_t)j * 16;
    const int i = j - k_pieces, d = i / pieces;
    return v0 + ((size_t)d * P + (i - d * pieces) * PER) * ES;
  };
  for (int j0 = threadIdx.x; j0 < all; j0 += 4 * 256) {
    u32x4 v[4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (j0 + x * 256 < all) v[x] = *(const u32x4 *)(src + offset(j0 + x * 256));
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int j = j0 + x * 256;
      if (j >= all) continue;
      char *const to_v = dst + offset(j);
      const int left = j < k_pieces ? PER : n - (j - k_pieces) % pieces * PER;         // tokens of the piece that are there
      if (left >= PER) {
        *(u32x4 *)to_v = v[x];
      } else {
#pragma unroll
        for (int e = 0; e < PER; ++e)
          if (e < left) ((T *)to_v)[e] = ((const T *)&v[x])[e];
      }
    }
  }
}

void kv_fork(hipStream_t s, const ForkArgs &a) {
  k_fork_rows<<<a.n_old + a.n_new, 256, 0, s>>>(a);
  if (a.n_new == 0) return;
  k_fork_pages<<<1, 1024, 0, s>>>(a);
  const dim3 grid(a.n_new * a.g.n_kv_heads, a.g.n_layers);
  a.dtype == FOCUS_F32 ? k_fork_copy<4><<<grid, 256, 0, s>>>(a) : k_fork_copy<2><<<grid, 256, 0, s>>>(a);
}

// Work buffers of a reservation: pages wanted by the rows before, pages held, pages wanted at all.
__global__ __launch_bounds__(64) void k_reserve_rows(ReserveArgs a) {
  const int b = blockIdx.x;
  const int held = held_pages(a.table + (size_t)b * a.stride, a.stride);
  if (threadIdx.x == 0) {
    const int64_t need = ((int64_t)max(a.lens[b], 0) + a.room + a.page_size - 1) / a.page_size, wants = max(need - held, (int64_t)0);
    a.work[b] = (int)min(wants, (int64_t)(a.stride - held));
    a.work[a.n_seq + 1 + b] = held;
    a.work[2 * (size_t)a.n_seq + 1 + b] = (int)wants;
  }
}

__global__ __launch_bounds__(1024) void k_reserve_pages(ReserveArgs a) {
  __shared__ int part[16];
  __shared__ int start_s[kWantsInLds];                 // where a row's wants begin, looked up here for up to so many rows
  int32_t *const start = a.work, *const held = a.work + a.n_seq + 1, *const wants = a.work + 2 * (size_t)a.n_seq + 1;
  const bool in_lds = a.n_seq <= kWantsInLds;
  const int wanted = order_wants(start, a.n_seq, part, [&](int b, int, int before) {
    if (in_lds) start_s[b] = before;
  });
  const int got = hand_out(a.refs, a.n_pages, wanted, part, [&](int rank, int page) {
    const int b = in_lds ? sequence_of(start_s, a.n_seq, rank) : sequence_of(start, a.n_seq, rank);
    a.table[(size_t)b * a.stride + held[b] + rank - (in_lds ? start_s[b] : start[b])] = page;
  });
  for (int b = threadIdx.x; b < a.n_seq; b += blockDim.x) a.lacking[b] = wants[b] - max(0, min(got, start[b + 1]) - start[b]);
}

void kv_reserve(hipStream_t s, const ReserveArgs &a) {
  k_reserve_rows<<<a.n_seq, 64, 0, s>>>(a);
  k_reserve_pages<<<1, 1024, 0, s>>>(a);
}

}  // namespace fk
