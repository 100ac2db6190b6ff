// C entries of the operators for generation that branches over the paged cache: argument checks and launches.
#include <math.h>

#include <initializer_list>

#include "focus_branch.h"

using fk::fail_call;

namespace {

bool aligned(const void *p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
// Of bytes.
bool overlap(const void *p, int64_t np, const void *q, int64_t nq) {
  return p && q && np > 0 && nq > 0 && (uintptr_t)p < (uintptr_t)q + (uintptr_t)nq && (uintptr_t)q < (uintptr_t)p + (uintptr_t)np;
}
struct List {            // of a call
  const void *p;
  int64_t bytes;
  bool written;
};
// Whether one that is written overlaps another.
bool collide(std::initializer_list<List> lists) {
  for (const List *x = lists.begin(); x != lists.end(); ++x)
    for (const List *y = x + 1; y != lists.end(); ++y)
      if ((x->written || y->written) && overlap(x->p, x->bytes, y->p, y->bytes)) return true;
  return false;
}

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? FOCUS_OK : fail_call(FOCUS_EHIP, "launch: %s", hipGetErrorString(e));
}

constexpr int kMaxRows = 1 << 20;            // rows of a page table
constexpr int kMaxPages = 1 << 30;           // of a pool

int esize(int dtype) { return dtype == FOCUS_F32 ? 4 : 2; }

const char *check_kv(const focus_kv *kv) {
  if (!kv) return "null kv";
  if (kv->dtype != FOCUS_F32 && kv->dtype != FOCUS_BF16) return "dtype of the pool must be FOCUS_F32 or FOCUS_BF16";
  if (kv->head_dim != 64 && kv->head_dim != 128) return "head_dim must be 64 or 128";
  if (kv->page_size < 8 || kv->page_size > 1024 || kv->page_size % 8) return "page_size must be a multiple of 8 in 8..1024";
  if (kv->n_kv_heads < 1 || kv->n_kv_heads > 256) return "n_kv_heads must be in 1..256";
  if (kv->n_layers < 1 || kv->n_layers > 1024) return "n_layers must be in 1..1024";
  if (kv->n_pages < 1 || kv->n_pages > kMaxPages) return "n_pages must be in 1..2^30";
  return nullptr;
}
const char *check_pool(const focus_kv *kv) {
  if (!kv->pool) return "null pool";
  return aligned(kv->pool, 16) ? nullptr : "the pool must be 16-byte aligned";
}

fk::Paged paged(const focus_kv &kv, int layer, const int32_t *table, int stride) {
  const size_t layer_bytes = (size_t)kv.n_pages * 2 * kv.n_kv_heads * kv.page_size * kv.head_dim * esize(kv.dtype);
  return fk::Paged{(char *)kv.pool + layer_bytes * layer, kv.n_pages, kv.page_size, kv.n_kv_heads, kv.n_layers, table, stride};
}

// What append and attention have in common.
const char *check_rows(const focus_kv *kv, int32_t layer, int32_t n_seq, int32_t n_rows, int32_t table_stride) {
  if (const char *e = check_kv(kv)) return e;
  if (layer < 0 || layer >= kv->n_layers) return "no such layer";
  if (n_seq < 0 || n_seq >= kMaxRows) return "n_seq must be in 0..2^20 - 1";
  if (n_rows < 0 || n_rows > (1 << 22)) return "n_rows must be in 0..2^22";
  if (table_stride < 1) return "table_stride must be positive";
  return nullptr;
}

const char *check_tree(const focus_kv *kv, int32_t n_seq, int32_t n_rows, int32_t max_rows, int32_t max_len, int32_t table_stride, int32_t n_q_heads) {
  if (const char *e = check_rows(kv, 0, n_seq, n_rows, table_stride)) return e;
  if (n_q_heads < 1 || n_q_heads > 1024 || n_q_heads % kv->n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads, at most 1024";
  if ((int64_t)n_rows * n_q_heads >= (1ll << 31)) return "n_rows * n_q_heads must be below 2^31";
  if (max_rows < 0 || max_len < 0) return "max_rows and max_len must not be negative";
  return nullptr;
}

fk::TreeArgs tree_args(const focus_kv *kv, int32_t layer, int32_t n_seq, int32_t n_rows, int32_t max_rows, int32_t max_len, const int32_t *page_table,
                       int32_t table_stride, int32_t n_q_heads) {
  fk::TreeArgs a{};
  a.dtype = kv->dtype; a.head_dim = kv->head_dim; a.g = paged(*kv, layer, page_table, table_stride);
  a.n_seq = n_seq; a.n_rows = n_rows; a.n_q_heads = n_q_heads; a.max_rows = max_rows; a.max_len = max_len;
  return a;
}

}  // namespace

extern "C" {

int focus_kv_append(const focus_kv *kv, void *hip_stream, int32_t layer, int32_t n_seq, int32_t n_rows, const int32_t *cu_rows, const int32_t *lens,
                    const int32_t *page_table, int32_t table_stride, const void *k, int64_t ldk, const void *v, int64_t ldv) {
  if (const char *e = check_rows(kv, layer, n_seq, n_rows, table_stride)) return fail_call(FOCUS_EINVAL, "%s", e);
  const int64_t width = (int64_t)kv->n_kv_heads * kv->head_dim;
  if (ldk < width || ldv < width) return fail_call(FOCUS_EINVAL, "ldk and ldv must be at least n_kv_heads * head_dim");
  if (n_seq == 0 || n_rows == 0) return FOCUS_OK;
  if (const char *e = check_pool(kv)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (!cu_rows || !lens || !page_table || !k || !v) return fail_call(FOCUS_EINVAL, "null operand");
  if (!aligned(cu_rows, 4) || !aligned(lens, 4) || !aligned(page_table, 4) || !aligned(k, esize(kv->dtype)) || !aligned(v, esize(kv->dtype)))
    return fail_call(FOCUS_EINVAL, "a pointer is not aligned to its elements");
  fk::AppendArgs a{};
  a.dtype = kv->dtype; a.head_dim = kv->head_dim; a.g = paged(*kv, layer, page_table, table_stride);
  a.n_seq = n_seq; a.n_rows = n_rows; a.cu = cu_rows; a.lens = lens; a.k = k; a.v = v; a.ldk = ldk; a.ldv = ldv;
  fk::kv_append((hipStream_t)hip_stream, a);
  return launched();
}

int focus_tree_attention_bytes(const focus_kv *kv, int32_t n_seq, int32_t n_rows, int32_t max_rows, int32_t max_len, int32_t table_stride, int32_t n_q_heads, size_t *bytes) {
  if (!bytes) return fail_call(FOCUS_EINVAL, "null bytes");
  if (const char *e = check_tree(kv, n_seq, n_rows, max_rows, max_len, table_stride, n_q_heads)) return fail_call(FOCUS_EINVAL, "%s", e);
  *bytes = n_seq > 0 && n_rows > 0 ? fk::tree_scratch(tree_args(kv, 0, n_seq, n_rows, max_rows, max_len, nullptr, table_stride, n_q_heads)) : 0;
  return FOCUS_OK;
}

int focus_tree_attention(const focus_kv *kv, void *hip_stream, int32_t layer, int32_t n_seq, int32_t n_rows, int32_t max_rows, int32_t max_len, const int32_t *cu_rows,
                         const int32_t *lens, const int32_t *page_table, int32_t table_stride, const uint64_t *seen, int32_t seen_words, int32_t n_q_heads,
                         float scale, const void *q, int64_t ldq, void *out, int64_t ldo, void *workspace, size_t workspace_bytes) {
  if (const char *e = check_tree(kv, n_seq, n_rows, max_rows, max_len, table_stride, n_q_heads)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (layer < 0 || layer >= kv->n_layers) return fail_call(FOCUS_EINVAL, "no such layer");
  if (seen && (seen_words < 1 || seen_words > 16)) return fail_call(FOCUS_EINVAL, "seen_words must be in 1..16");
  if (!isfinite(scale)) return fail_call(FOCUS_EINVAL, "scale must be finite");
  const int64_t width = (int64_t)n_q_heads * kv->head_dim;
  if (ldq < width || ldo < width) return fail_call(FOCUS_EINVAL, "ldq and ldo must be at least n_q_heads * head_dim");
  if (n_seq == 0 || n_rows == 0) return FOCUS_OK;
  if (const char *e = check_pool(kv)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (!cu_rows || !lens || !page_table || !q || !out) return fail_call(FOCUS_EINVAL, "null operand");
  if (!aligned(cu_rows, 4) || !aligned(lens, 4) || !aligned(page_table, 4) || !aligned(seen, 8) || !aligned(q, esize(kv->dtype)) || !aligned(out, esize(kv->dtype)))
    return fail_call(FOCUS_EINVAL, "a pointer is not aligned to its elements");
  if (!aligned(workspace, 256)) return fail_call(FOCUS_EINVAL, "the workspace must be 256-byte aligned");
  fk::TreeArgs a = tree_args(kv, layer, n_seq, n_rows, max_rows, max_len, page_table, table_stride, n_q_heads);
  a.cu = cu_rows; a.lens = lens; a.seen = seen; a.seen_words = seen ? seen_words : 0; a.scale = scale; a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo;
  a.scratch = fk::Scratch{workspace, workspace ? workspace_bytes : 0};
  fk::tree_attention((hipStream_t)hip_stream, a);
  return launched();
}

int focus_kv_compact(const focus_kv *kv, void *hip_stream, int32_t n_seq, int32_t n_keep, const int32_t *start, const int32_t *cu_keep, const int32_t *keep, const int32_t *page_table,
                     int32_t table_stride, const int32_t *to_table, int32_t to_stride) {
  if (const char *e = check_rows(kv, 0, n_seq, 0, table_stride)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (n_keep < 0 || n_keep > (1 << 30)) return fail_call(FOCUS_EINVAL, "n_keep must be in 0..2^30");
  if (to_stride < 1) return fail_call(FOCUS_EINVAL, "to_stride must be positive");
  if ((int64_t)n_seq * kv->n_kv_heads * kv->n_layers >= fk::kMaxGroups) return fail_call(FOCUS_EINVAL, "n_seq * n_kv_heads * n_layers must be below 2^24");
  if (n_seq == 0 || n_keep == 0) return FOCUS_OK;
  if (const char *e = check_pool(kv)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (!start || !cu_keep || !keep || !page_table || !to_table) return fail_call(FOCUS_EINVAL, "null operand");
  if (!aligned(start, 4) || !aligned(cu_keep, 4) || !aligned(keep, 4) || !aligned(page_table, 4) || !aligned(to_table, 4)) return fail_call(FOCUS_EINVAL, "a pointer is not aligned to its elements");
  fk::CompactArgs a{};
  a.dtype = kv->dtype; a.head_dim = kv->head_dim; a.g = paged(*kv, 0, page_table, table_stride);
  a.n_seq = n_seq; a.n_keep = n_keep; a.start = start; a.cu = cu_keep; a.keep = keep; a.to_table = to_table; a.to_stride = to_stride;
  fk::kv_compact((hipStream_t)hip_stream, a);
  return launched();
}

int focus_kv_fork_bytes(int32_t n_new, size_t *bytes) {
  if (!bytes) return fail_call(FOCUS_EINVAL, "null bytes");
  if (n_new < 0 || n_new >= kMaxRows) return fail_call(FOCUS_EINVAL, "n_new must be in 0..2^20 - 1");
  *bytes = 4 * fk::fork_ints(n_new);
  return FOCUS_OK;
}

int focus_kv_fork(const focus_kv *kv, void *hip_stream, int32_t n_old, int32_t n_new, const int32_t *parents, const int32_t *lens, const int32_t *page_table,
                  int32_t table_stride, int32_t *new_lens, int32_t *new_table, int32_t *refs, int32_t *lacking, void *workspace, size_t workspace_bytes) {
  if (const char *e = check_kv(kv)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (n_old < 0 || n_new < 0 || n_old >= kMaxRows || n_new >= kMaxRows - n_old) return fail_call(FOCUS_EINVAL, "n_old and n_new must not be negative and be below 2^20 together");
  if (table_stride < 1 || (int64_t)(n_old + n_new) * table_stride >= (1ll << 31)) return fail_call(FOCUS_EINVAL, "table_stride must be positive and (n_old + n_new) * table_stride below 2^31");
  if ((int64_t)n_new * kv->n_kv_heads * kv->n_layers >= fk::kMaxGroups) return fail_call(FOCUS_EINVAL, "n_new * n_kv_heads * n_layers must be below 2^24");
  if (n_old + n_new == 0) return FOCUS_OK;
  if (const char *e = check_pool(kv)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (!refs || (n_old > 0 && (!lens || !page_table)) || (n_new > 0 && (!parents || !new_lens || !new_table || !lacking || !workspace))) return fail_call(FOCUS_EINVAL, "null operand");
  if (!aligned(parents, 4) || !aligned(lens, 4) || !aligned(page_table, 4) || !aligned(new_lens, 4) || !aligned(new_table, 4) || !aligned(refs, 4) || !aligned(lacking, 4) || !aligned(workspace, 16))
    return fail_call(FOCUS_EINVAL, "the workspace must be 16-byte aligned, the others to their elements");
  if (new_table && (const int32_t *)new_table == page_table) return fail_call(FOCUS_EINVAL, "new_table must not be page_table");
  if (n_new > 0 && workspace_bytes < 4 * fk::fork_ints(n_new)) return fail_call(FOCUS_ENOMEM, "the workspace is too small");
  // Workgroups read all of the inputs, and the counts, while others write the outputs.
  const int64_t old_bytes = 4 * (int64_t)n_old, new_bytes = 4 * (int64_t)n_new;
  if (collide({{new_lens, new_bytes, true}, {new_table, new_bytes * table_stride, true}, {lacking, new_bytes, true}, {refs, 4 * (int64_t)kv->n_pages, true},
               {workspace, n_new > 0 ? 4 * (int64_t)fk::fork_ints(n_new) : 0, true}, {parents, new_bytes, false}, {lens, old_bytes, false}, {page_table, old_bytes * table_stride, false}}))
    return fail_call(FOCUS_EINVAL, "outputs, refs and the workspace must overlap neither an input nor each other");
  fk::ForkArgs a{};
  a.dtype = kv->dtype; a.head_dim = kv->head_dim; a.g = paged(*kv, 0, page_table, table_stride);
  a.n_old = n_old; a.n_new = n_new; a.parents = parents; a.lens = lens; a.new_lens = new_lens; a.new_table = new_table; a.refs = refs; a.lacking = lacking;
  a.work = (int32_t *)workspace;
  fk::kv_fork((hipStream_t)hip_stream, a);
  return launched();
}

int focus_kv_reserve_bytes(int32_t n_seq, size_t *bytes) {
  if (!bytes) return fail_call(FOCUS_EINVAL, "null bytes");
  if (n_seq < 0 || n_seq >= kMaxRows) return fail_call(FOCUS_EINVAL, "n_seq must be in 0..2^20 - 1");
  *bytes = 4 * fk::reserve_ints(n_seq);
  return FOCUS_OK;
}

int focus_kv_reserve(void *hip_stream, int32_t n_seq, int32_t page_size, int32_t n_pages, const int32_t *lens, int32_t room, int32_t *page_table, int32_t table_stride,
                     int32_t *refs, int32_t *lacking, void *workspace, size_t workspace_bytes) {
  if (n_seq < 0 || n_seq >= kMaxRows) return fail_call(FOCUS_EINVAL, "n_seq must be in 0..2^20 - 1");
  if (page_size < 8 || page_size > 1024 || page_size % 8) return fail_call(FOCUS_EINVAL, "page_size must be a multiple of 8 in 8..1024");
  if (n_pages < 1 || n_pages > kMaxPages) return fail_call(FOCUS_EINVAL, "n_pages must be in 1..2^30");
  if (table_stride < 1 || (int64_t)n_seq * table_stride >= (1ll << 31)) return fail_call(FOCUS_EINVAL, "table_stride must be positive and n_seq * table_stride below 2^31");
  if (room < 0) return fail_call(FOCUS_EINVAL, "room must not be negative");
  if (n_seq == 0) return FOCUS_OK;
  if (!lens || !page_table || !refs || !lacking || !workspace) return fail_call(FOCUS_EINVAL, "null operand");
  if (!aligned(lens, 4) || !aligned(page_table, 4) || !aligned(refs, 4) || !aligned(lacking, 4) || !aligned(workspace, 16))
    return fail_call(FOCUS_EINVAL, "the workspace must be 16-byte aligned, the others to their elements");
  if (workspace_bytes < 4 * fk::reserve_ints(n_seq)) return fail_call(FOCUS_ENOMEM, "the workspace is too small");
  // Lengths are read by the first launch and `lacking` is written by the second.
  const List table = {page_table, 4 * (int64_t)n_seq * table_stride, true}, counts = {refs, 4 * (int64_t)n_pages, true}, work = {workspace, 4 * (int64_t)fk::reserve_ints(n_seq), true};
  if (collide({table, counts, work, {lens, 4 * (int64_t)n_seq, false}}) || collide({table, counts, work, {lacking, 4 * (int64_t)n_seq, true}}))
    return fail_call(FOCUS_EINVAL, "page_table, refs, lacking and the workspace must not overlap each other, nor lens any but lacking");
  fk::ReserveArgs a{};
  a.n_seq = n_seq; a.page_size = page_size; a.n_pages = n_pages; a.room = room; a.stride = table_stride; a.lens = lens; a.table = page_table; a.refs = refs;
  a.lacking = lacking; a.work = (int32_t *)workspace;
  fk::kv_reserve((hipStream_t)hip_stream, a);
  return launched();
}

static const char *check_beams(int32_t n_seq, int32_t n_beams, int32_t vocab, int32_t k) {
  if (n_beams < 1 || n_beams > fk::kMaxBeams || k < 1 || k > fk::kMaxPicks) return "n_beams and k must be in 1..64";
  if (n_seq < 0 || (int64_t)n_seq * n_beams > kMaxRows) return "n_seq must not be negative and n_seq * n_beams at most 2^20";
  if (vocab < 1 || vocab > (1 << 24)) return "vocab must be in 1..2^24";
  if (fk::beam_groups(n_seq, n_beams, vocab, k) >= fk::kMaxGroups) return "n_seq, n_beams and vocab too large";
  return nullptr;
}

int focus_beam_select_bytes(int32_t n_seq, int32_t n_beams, int32_t vocab, int32_t k, size_t *bytes) {
  if (!bytes) return fail_call(FOCUS_EINVAL, "null bytes");
  if (const char *e = check_beams(n_seq, n_beams, vocab, k)) return fail_call(FOCUS_EINVAL, "%s", e);
  *bytes = n_seq > 0 ? fk::beam_scratch(n_seq, n_beams, vocab, k) : 0;
  return FOCUS_OK;
}

int focus_beam_select(void *hip_stream, int32_t n_seq, int32_t n_beams, int32_t vocab, int32_t k, int32_t dtype, const void *logits, int64_t ld, const float *scores,
                      const uint8_t *done, int32_t end_token, int32_t *rows, int32_t *tokens, float *new_scores, void *workspace, size_t workspace_bytes) {
  if (const char *e = check_beams(n_seq, n_beams, vocab, k)) return fail_call(FOCUS_EINVAL, "%s", e);
  if (dtype != FOCUS_F32 && dtype != FOCUS_BF16) return fail_call(FOCUS_EINVAL, "dtype must be FOCUS_F32 or FOCUS_BF16");
  if (ld < vocab) return fail_call(FOCUS_EINVAL, "ld is less than vocab");
  if (n_seq == 0) return FOCUS_OK;
  if (!logits || !scores || !rows || !tokens || !new_scores || !workspace) return fail_call(FOCUS_EINVAL, "null operand");
  if (!aligned(logits, esize(dtype)) || !aligned(scores, 4) || !aligned(rows, 4) || !aligned(tokens, 4) || !aligned(new_scores, 4) || !aligned(workspace, 256))
    return fail_call(FOCUS_EINVAL, "the workspace must be 256-byte aligned, the others to their elements");
  if (workspace_bytes < fk::beam_scratch(n_seq, n_beams, vocab, k)) return fail_call(FOCUS_ENOMEM, "the workspace is too small");
  // A request's workgroup reads its own scores and done before it writes its picks, but not before others write theirs.
  const int64_t picks = 4 * (int64_t)n_seq * k, beams = (int64_t)n_seq * n_beams, work = (int64_t)fk::beam_scratch(n_seq, n_beams, vocab, k);
  for (const void *out : {(const void *)rows, (const void *)tokens, (const void *)new_scores})
    if (!(out == scores && k == n_beams) && overlap(out, picks, scores, 4 * beams))
      return fail_call(FOCUS_EINVAL, "new_scores may be scores where k is n_beams and must not overlap them otherwise, nor may another output");
  if (collide({{rows, picks, true}, {tokens, picks, true}, {new_scores, picks, true}, {workspace, work, true}, {done, beams, false}}) || overlap(workspace, work, scores, 4 * beams))
    return fail_call(FOCUS_EINVAL, "outputs and the workspace must overlap neither an input nor each other");
  fk::BeamArgs a{};
  a.n_seq = n_seq; a.n_beams = n_beams; a.vocab = vocab; a.k = k; a.dtype = dtype; a.logits = logits; a.ld = ld; a.scores = scores; a.done = done; a.end_token = end_token;
  a.rows = rows; a.tokens = tokens; a.new_scores = new_scores; a.work = workspace;
  fk::beam_select((hipStream_t)hip_stream, a);
  return launched();
}

}  // extern "C"
