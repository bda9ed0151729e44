// Host side of the operators on the caller's tensors (tss.h): argument checks
// and launches.  Nothing is kept between calls.
#include "../../include/tss.h"
#include "tss_internal.h"

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <vector>

using namespace tss;

namespace {

int refuse(int code, const char* where, const char* msg) {
  char b[256];
  std::snprintf(b, sizeof(b), "%s: %s", where, msg);
  set_thread_error(b);
  return code;
}

int launched(hipError_t e, const char* where) {
  return e == hipSuccess ? TSS_OK : refuse(TSS_EHIP, where, hipGetErrorString(e));
}

int type_size(int32_t t) { return t == TSS_T_F32 ? 4 : (t == TSS_T_BF16 || t == TSS_T_F16) ? 2 : 0; }

bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// What is wrong with the sizes of a call, or null.
const char* logprobs_fault(int32_t rows, int32_t vocab, int32_t n_tokens, int32_t top_k) {
  if (rows < 0 || vocab < 1) return "bad rows or vocab";
  if (n_tokens < 0 || n_tokens > TSS_LOGPROBS_MAX_TOKENS || top_k < 0 || top_k > TSS_LOGPROBS_MAX_TOP || top_k > vocab)
    return "n_tokens outside [0, 8] or top_k outside [0, min(32, vocab)]";
  if (!logprobs_fit(rows, vocab)) return "more than 2^20 tokens in the vocabulary, or too many rows for one launch";
  return nullptr;
}

// What is wrong with a cache's description, or null.
const char* kv_fault(const tss_paged_kv* kv) {
  if (!kv || !kv->pages) return "no cache";
  if (kv->type != TSS_T_F32 && kv->type != TSS_T_F16) return "the cache's type must be TSS_T_F32 or TSS_T_F16";
  if (kv->head_dim != 64 && kv->head_dim != 128) return "head_dim must be 64 or 128";
  if (kv->n_layers < 1 || kv->n_pages < 1 || kv->n_kv_heads < 1 || kv->n_kv_heads > 65535)
    return "layers, pages and heads must be positive (heads up to 65535)";
  if (kv->n_layers > kMaxLayers) return "too many layers";
  if (!aligned(kv->pages, 16)) return "pages must be aligned to 16 bytes";
  return nullptr;
}

const char* table_fault(const tss_paged_kv* kv) {
  return kv->n_seqs < 0 || kv->table_stride < 1 || kv->table_stride > INT32_MAX / kPage ? "bad page table" : nullptr;
}

const char* window_fault(const tss_paged_kv* kv, int32_t n_q_heads, int32_t rows, int32_t max_rows, int32_t max_length,
                         int32_t sinks, int32_t window) {
  if (const char* f = table_fault(kv)) return f;
  if (n_q_heads < 1 || n_q_heads % kv->n_kv_heads) return "n_q_heads must be a multiple of n_kv_heads";
  if (rows < 0 || max_rows < 0 || max_length < 0 || sinks < 0 || window < 0)
    return "negative rows, length, sinks or window";
  if (sinks > INT32_MAX - kPage) return "too many sinks";
  if (!window_fits(kv->n_kv_heads, n_q_heads / kv->n_kv_heads, kv->n_seqs, std::min(max_rows, rows)))
    return "too many sequences, heads or rows for one launch";
  return nullptr;
}

const char* prefix_fault(const tss_paged_kv* kv, int32_t n_q_heads, int32_t rows, int32_t max_rows, int32_t max_length,
                         int32_t n_groups, int32_t max_group_rows, int32_t max_shared) {
  if (const char* f = window_fault(kv, n_q_heads, rows, max_rows, max_length, 0, 0)) return f;
  if (n_groups < 0 || max_group_rows < 0 || max_shared < 0) return "negative groups, rows of a group or shared pages";
  if (!prefix_fits(kv->n_kv_heads, n_q_heads / kv->n_kv_heads, kv->n_seqs, std::min(max_rows, rows), n_groups,
                   std::min(max_group_rows, rows)))
    return "too many groups or rows of a group for one launch";
  return nullptr;
}

const char* beams_fault(int32_t n_groups, int32_t n_beams, int32_t vocab, int32_t n) {
  if (n_groups < 0 || vocab < 1) return "bad n_groups or vocab";
  if (n_beams < 1 || n_beams > TSS_BEAMS_MAX) return "n_beams outside [1, 32]";
  if (n < 1 || n > TSS_BEAMS_MAX_N || n > (int64_t)n_beams * vocab) return "n outside [1, min(64, n_beams * vocab)]";
  if (!beams_fit(n_groups, n_beams, vocab))
    return "more than 2^20 tokens in the vocabulary, or too many beams for one launch";
  return nullptr;
}

size_t page_bytes(const tss_paged_kv* kv) {
  return (size_t)2 * kv->n_kv_heads * kPage * kv->head_dim * type_size(kv->type);
}

uint8_t* layer_pages(const tss_paged_kv* kv, int32_t layer) {
  return (uint8_t*)kv->pages + (size_t)layer * kv->n_pages * page_bytes(kv);
}

// Fills in what the attention calls have in common; returns what is wrong with it, or null.
// a->rows = 0: nothing to launch.
const char* rows_fault(WindowArgs* a, const tss_paged_kv* kv, int32_t layer, const void* q, int64_t q_stride,
                       int32_t n_q_heads, int32_t rows, int32_t max_rows, float scale, void* out, int64_t out_stride) {
  // in powers of two, as the kernels take it
  const float scale_log2 =
      (float)(1.4426950408889634 * (scale > 0.f ? (double)scale : 1.0 / std::sqrt((double)kv->head_dim)));
  if (!(scale >= 0.f) || std::isinf(scale_log2))
    return "scale must be finite (its product with log2 e too) and not negative";
  if (rows == 0 || max_rows == 0 || kv->n_seqs == 0) return nullptr;
  const int64_t width = (int64_t)n_q_heads * kv->head_dim;
  if (q_stride < width || out_stride < width || q_stride % 8 || out_stride % 8)
    return "q_stride and out_stride must be multiples of 8 that hold every head";
  if (!aligned(q, 16) || !aligned(out, 16)) return "q and out must be aligned to 16 bytes";
  a->q = q;
  a->o = out;
  a->q_stride = q_stride;
  a->o_stride = out_stride;
  a->kv_pages = layer_pages(kv, layer);
  a->page_table = kv->page_table;
  a->n_pages = kv->n_pages;
  a->n_heads = kv->n_kv_heads;
  a->group = n_q_heads / kv->n_kv_heads;
  a->n_seqs = kv->n_seqs;
  a->table_stride = kv->table_stride;
  a->rows = rows;
  a->max_rows = std::min(max_rows, rows);
  a->scale_log2 = scale_log2;
  return nullptr;
}

}  // namespace

extern "C" {

size_t tss_token_logprobs_bytes(int32_t rows, int32_t vocab, int32_t n_tokens, int32_t top_k) {
  return logprobs_fault(rows, vocab, n_tokens, top_k) ? 0 : logprobs_bytes(rows, vocab, n_tokens, top_k);
}

int tss_token_logprobs(void* hip_stream, const void* logits, int32_t type, int64_t row_stride, int32_t rows,
                       int32_t vocab, const int32_t* tokens, int32_t n_tokens, int32_t top_k, float* logprob,
                       int32_t* rank, float* entropy, float* top_logprob, int32_t* top_token, void* workspace,
                       size_t workspace_bytes) {
  const char* me = "tss_token_logprobs";
  const int es = type_size(type);
  if (!es) return refuse(TSS_EINVAL, me, "unknown element type");
  if (const char* f = logprobs_fault(rows, vocab, n_tokens, top_k)) return refuse(TSS_EINVAL, me, f);
  if (row_stride < vocab) return refuse(TSS_EINVAL, me, "row_stride smaller than vocab");
  if (rows == 0) return TSS_OK;
  if (!logits || (n_tokens > 0 && !tokens)) return refuse(TSS_EINVAL, me, "null tensor");
  if (!aligned(logits, es)) return refuse(TSS_EINVAL, me, "logits must be aligned to their elements");
  const size_t need = logprobs_bytes(rows, vocab, n_tokens, top_k);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16)))
    return refuse(TSS_ENOSPACE, me, "workspace smaller than tss_token_logprobs_bytes() or not aligned to 16 bytes");
  LogprobArgs a{};
  a.x = logits;
  a.stride = row_stride;
  a.rows = rows;
  a.vocab = vocab;
  a.type = type;
  a.tokens = tokens;
  a.n_tokens = n_tokens;
  a.top_k = top_k;
  a.logprob = logprob;
  a.rank = rank;
  a.entropy = entropy;
  a.top_logprob = top_logprob;
  a.top_token = top_token;
  return launched(launch_logprobs(a, workspace, (hipStream_t)hip_stream), me);
}

size_t tss_window_attn_bytes(const tss_paged_kv* kv, int32_t n_q_heads, int32_t rows, int32_t max_rows,
                             int32_t max_length, int32_t sinks, int32_t window) {
  if (kv_fault(kv) || window_fault(kv, n_q_heads, rows, max_rows, max_length, sinks, window)) return 0;
  max_rows = std::min(max_rows, rows);
  if (max_rows == 0 || kv->n_seqs == 0) return 0;
  return window_bytes(kv->type == TSS_T_F16, kv->head_dim, kv->n_kv_heads, n_q_heads / kv->n_kv_heads, kv->n_seqs, rows,
                      max_rows, std::min(max_length, kv->table_stride * kPage), sinks, window);
}

int tss_window_attn(void* hip_stream, const tss_paged_kv* kv, int32_t layer, const void* q, int64_t q_stride,
                    int32_t n_q_heads, const int32_t* row_offsets, const int32_t* lengths, int32_t rows,
                    int32_t max_rows, int32_t max_length, int32_t sinks, int32_t window, float scale, void* out,
                    int64_t out_stride, void* workspace, size_t workspace_bytes) {
  const char* me = "tss_window_attn";
  if (const char* f = kv_fault(kv)) return refuse(TSS_EINVAL, me, f);
  if (layer < 0 || layer >= kv->n_layers) return refuse(TSS_EINVAL, me, "no such layer");
  if (const char* f = window_fault(kv, n_q_heads, rows, max_rows, max_length, sinks, window))
    return refuse(TSS_EINVAL, me, f);
  WindowArgs a{};
  if (const char* f = rows_fault(&a, kv, layer, q, q_stride, n_q_heads, rows, max_rows, scale, out, out_stride))
    return refuse(TSS_EINVAL, me, f);
  if (a.rows == 0) return TSS_OK;
  if (!q || !out || !row_offsets || !lengths || !kv->page_table) return refuse(TSS_EINVAL, me, "null tensor");
  const size_t need = tss_window_attn_bytes(kv, n_q_heads, rows, max_rows, max_length, sinks, window);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16)))
    return refuse(TSS_ENOSPACE, me, "workspace smaller than tss_window_attn_bytes() or not aligned to 16 bytes");
  a.row_offsets = row_offsets;
  a.lengths = lengths;
  a.max_length = std::min(max_length, kv->table_stride * kPage);
  a.sinks = sinks;
  a.window = window;
  return launched(launch_window(kv->type == TSS_T_F16, kv->head_dim, a, workspace, (hipStream_t)hip_stream), me);
}

size_t tss_prefix_attn_bytes(const tss_paged_kv* kv, int32_t n_q_heads, int32_t rows, int32_t max_rows,
                             int32_t max_length, int32_t n_groups, int32_t max_group_rows, int32_t max_shared) {
  if (kv_fault(kv) || prefix_fault(kv, n_q_heads, rows, max_rows, max_length, n_groups, max_group_rows, max_shared))
    return 0;
  max_rows = std::min(max_rows, rows);
  if (max_rows == 0 || kv->n_seqs == 0) return 0;
  return prefix_bytes(kv->type == TSS_T_F16, kv->head_dim, kv->n_kv_heads, n_q_heads / kv->n_kv_heads, kv->n_seqs, rows,
                      max_rows, std::min(max_length, kv->table_stride * kPage), n_groups,
                      std::min(max_group_rows, rows), std::min(max_shared, kv->table_stride));
}

int tss_prefix_attn(void* hip_stream, const tss_paged_kv* kv, int32_t layer, const void* q, int64_t q_stride,
                    int32_t n_q_heads, const int32_t* row_offsets, const int32_t* lengths, int32_t rows,
                    int32_t max_rows, int32_t max_length, const int32_t* group_offsets, const int32_t* shared,
                    int32_t n_groups, int32_t max_group_rows, int32_t max_shared, float scale, void* out,
                    int64_t out_stride, void* workspace, size_t workspace_bytes) {
  const char* me = "tss_prefix_attn";
  if (const char* f = kv_fault(kv)) return refuse(TSS_EINVAL, me, f);
  if (layer < 0 || layer >= kv->n_layers) return refuse(TSS_EINVAL, me, "no such layer");
  if (const char* f = prefix_fault(kv, n_q_heads, rows, max_rows, max_length, n_groups, max_group_rows, max_shared))
    return refuse(TSS_EINVAL, me, f);
  PrefixArgs a{};
  if (const char* f = rows_fault(&a, kv, layer, q, q_stride, n_q_heads, rows, max_rows, scale, out, out_stride))
    return refuse(TSS_EINVAL, me, f);
  if (a.rows == 0) return TSS_OK;
  if (!q || !out || !row_offsets || !lengths || !kv->page_table || (n_groups > 0 && !shared) ||
      (n_groups > 1 && !group_offsets))
    return refuse(TSS_EINVAL, me, "null tensor");
  const size_t need =
      tss_prefix_attn_bytes(kv, n_q_heads, rows, max_rows, max_length, n_groups, max_group_rows, max_shared);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned(workspace, 16)))
    return refuse(TSS_ENOSPACE, me, "workspace smaller than tss_prefix_attn_bytes() or not aligned to 16 bytes");
  a.row_offsets = row_offsets;
  a.lengths = lengths;
  a.max_length = std::min(max_length, kv->table_stride * kPage);
  a.group_offsets = group_offsets;
  a.shared = shared;
  a.n_groups = n_groups;
  a.max_group_rows = std::min(max_group_rows, rows);
  a.max_shared = std::min(max_shared, kv->table_stride);
  return launched(launch_prefix(kv->type == TSS_T_F16, kv->head_dim, a, workspace, (hipStream_t)hip_stream), me);
}

int tss_append_kv(void* hip_stream, const tss_paged_kv* kv, int32_t layer, const void* q, int64_t q_stride,
                  int32_t n_q_heads, const void* k, int64_t k_stride, const void* v, int64_t v_stride, int32_t type,
                  const int32_t* row_offsets, const int32_t* lengths, const int32_t* positions, int32_t rows,
                  int32_t max_rows, const double* inv_freq, void* q_out, int64_t q_out_stride) {
  const char* me = "tss_append_kv";
  if (const char* f = kv_fault(kv)) return refuse(TSS_EINVAL, me, f);
  if (layer < 0 || layer >= kv->n_layers) return refuse(TSS_EINVAL, me, "no such layer");
  if (!type_size(type)) return refuse(TSS_EINVAL, me, "unknown element type");
  if (const char* f = table_fault(kv)) return refuse(TSS_EINVAL, me, f);
  if (n_q_heads < 0 || rows < 0 || max_rows < 0) return refuse(TSS_EINVAL, me, "negative heads or rows");
  max_rows = std::min(max_rows, rows);
  if (!append_fits(n_q_heads, kv->n_kv_heads, kv->n_seqs, max_rows))
    return refuse(TSS_EINVAL, me, "too many sequences, heads or rows for one launch");
  AppendArgs a{};
  if (inv_freq) {
    a.rotate = 1;
    for (int j = 0; j < kv->head_dim / 2; ++j) {
      // at a million radians a position, 2^31 positions leave 64 bits no fraction of a turn to speak of
      if (!(std::fabs(inv_freq[j]) <= 1e6)) return refuse(TSS_EINVAL, me, "a frequency is beyond 1e6 in size");
      a.turns[j] = inv_freq[j] / 6.283185307179586476925;
    }
  }
  if (max_rows == 0 || kv->n_seqs == 0) return TSS_OK;
  if (!k || !v || !row_offsets || !lengths || !kv->page_table || (n_q_heads > 0 && (!q || !q_out)))
    return refuse(TSS_EINVAL, me, "null tensor");
  const int64_t kw = (int64_t)kv->n_kv_heads * kv->head_dim, qw = (int64_t)n_q_heads * kv->head_dim;
  if (k_stride < kw || v_stride < kw || k_stride % 8 || v_stride % 8 ||
      (n_q_heads > 0 && (q_stride < qw || q_out_stride < qw || q_stride % 8 || q_out_stride % 8)))
    return refuse(TSS_EINVAL, me, "strides must be multiples of 8 that hold every head");
  if (!aligned(k, 16) || !aligned(v, 16) || (n_q_heads > 0 && (!aligned(q, 16) || !aligned(q_out, 16))))
    return refuse(TSS_EINVAL, me, "tensors must be aligned to 16 bytes");
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.kv_pages = layer_pages(kv, layer);
  a.page_table = kv->page_table;
  a.row_offsets = row_offsets;
  a.lengths = lengths;
  a.positions = positions;
  a.n_pages = kv->n_pages;
  a.n_heads = kv->n_kv_heads;
  a.n_q_heads = n_q_heads;
  a.n_seqs = kv->n_seqs;
  a.table_stride = kv->table_stride;
  a.rows = rows;
  a.max_rows = max_rows;
  a.type = type;
  return launched(launch_append(kv->type == TSS_T_F16, kv->head_dim, a, (hipStream_t)hip_stream), me);
}

size_t tss_beam_select_bytes(int32_t n_groups, int32_t n_beams, int32_t vocab, int32_t n) {
  return beams_fault(n_groups, n_beams, vocab, n) ? 0 : beams_bytes(n_groups, n_beams, vocab, n);
}

int tss_beam_select(void* hip_stream, const void* logits, int32_t type, int64_t row_stride, int32_t n_groups,
                    int32_t n_beams, int32_t vocab, const float* scores, const int32_t* ended, int32_t end_token,
                    int32_t n, float* score, int32_t* parent, int32_t* token, void* workspace,
                    size_t workspace_bytes) {
  const char* me = "tss_beam_select";
  const int es = type_size(type);
  if (!es) return refuse(TSS_EINVAL, me, "unknown element type");
  if (const char* f = beams_fault(n_groups, n_beams, vocab, n)) return refuse(TSS_EINVAL, me, f);
  if (row_stride < vocab) return refuse(TSS_EINVAL, me, "row_stride smaller than vocab");
  if (ended && (end_token < 0 || end_token >= vocab)) return refuse(TSS_EINVAL, me, "end_token outside the vocabulary");
  if (n_groups == 0) return TSS_OK;
  if (!logits || !scores || !score || !parent || !token) return refuse(TSS_EINVAL, me, "null tensor");
  if (!aligned(logits, es)) return refuse(TSS_EINVAL, me, "logits must be aligned to their elements");
  if (!workspace || workspace_bytes < beams_bytes(n_groups, n_beams, vocab, n) || !aligned(workspace, 16))
    return refuse(TSS_ENOSPACE, me, "workspace smaller than tss_beam_select_bytes() or not aligned to 16 bytes");
  BeamArgs a{};
  a.x = logits;
  a.stride = row_stride;
  a.n_groups = n_groups;
  a.n_beams = n_beams;
  a.vocab = vocab;
  a.type = type;
  a.scores = scores;
  a.ended = ended;
  a.end_token = end_token;
  a.n = n;
  a.score = score;
  a.parent = parent;
  a.token = token;
  return launched(launch_beams(a, workspace, (hipStream_t)hip_stream), me);
}

int tss_reorder_pages(void* hip_stream, const tss_paged_kv* kv, const int32_t* parents, int32_t n_beams,
                      const int32_t* lengths, const int32_t* shared, int32_t max_own) {
  const char* me = "tss_reorder_pages";
  if (const char* f = kv_fault(kv)) return refuse(TSS_EINVAL, me, f);
  if (const char* f = table_fault(kv)) return refuse(TSS_EINVAL, me, f);
  if (n_beams < 1 || n_beams > TSS_BEAMS_MAX || kv->n_seqs % n_beams)
    return refuse(TSS_EINVAL, me, "n_beams outside [1, 32], or sequences that are no multiple of it");
  if (max_own < 0) return refuse(TSS_EINVAL, me, "negative max_own");
  if (kv->n_seqs == 0 || max_own == 0) return TSS_OK;
  if (!parents || !lengths || !kv->page_table) return refuse(TSS_EINVAL, me, "null tensor");
  ReorderArgs a{};
  a.pages = (uint8_t*)kv->pages;
  a.page_bytes = page_bytes(kv);
  a.layer_bytes = a.page_bytes * kv->n_pages;
  a.n_layers = kv->n_layers;
  std::fill(a.layers, a.layers + kMaxLayers / 64, ~0ull);
  a.page_table = kv->page_table;
  a.parents = parents;
  a.lengths = lengths;
  a.shared = shared;
  a.n_pages = kv->n_pages;
  a.n_groups = kv->n_seqs / n_beams;
  a.n_beams = n_beams;
  a.table_stride = kv->table_stride;
  a.max_own = std::min(max_own, kv->table_stride * kPage);
  if (!reorder_fits(a)) return refuse(TSS_EINVAL, me, "too many groups or pages for one launch");
  return launched(launch_reorder(a, (hipStream_t)hip_stream), me);
}

int tss_copy_pages(void* hip_stream, const tss_paged_kv* kv, const int32_t* src, const int32_t* dst, int32_t n) {
  const char* me = "tss_copy_pages";
  if (const char* f = kv_fault(kv)) return refuse(TSS_EINVAL, me, f);
  if (n < 0 || (n > 0 && (!src || !dst))) return refuse(TSS_EINVAL, me, "bad list of pages");
  CopyArgs a{};
  a.pages = (uint8_t*)kv->pages;
  a.page_bytes = page_bytes(kv);
  a.layer_bytes = a.page_bytes * kv->n_pages;
  a.n_layers = kv->n_layers;
  std::fill(a.layers, a.layers + kMaxLayers / 64, ~0ull);
  try {
    std::vector<uint8_t> use(kv->n_pages, 0);  // 1: a source, 2: a destination
    for (int i = 0; i < n; ++i) {
      if (src[i] < 0 || src[i] >= kv->n_pages || dst[i] < 0 || dst[i] >= kv->n_pages)
        return refuse(TSS_EINVAL, me, "page outside the pool");
      use[src[i]] |= 1;
      if (use[dst[i]] & 2) return refuse(TSS_EINVAL, me, "a page is the destination of two copies");
      use[dst[i]] |= 2;
    }
    for (int i = 0; i < n; ++i)
      if (use[src[i]] == 3) return refuse(TSS_EINVAL, me, "a page is source and destination");
    // copies of one source next to each other: it is read once for them
    std::vector<int32_t> order(n);
    for (int i = 0; i < n; ++i) order[i] = i;
    std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) { return src[x] < src[y]; });
    for (int i0 = 0; i0 < n; i0 += kCopyPairs) {
      a.n = std::min(n - i0, kCopyPairs);
      for (int i = 0; i < a.n; ++i) {
        a.src[i] = src[order[i0 + i]];
        a.dst[i] = dst[order[i0 + i]];
      }
      if (const int r = launched(launch_copy_pages(a, (hipStream_t)hip_stream), me)) return r;
    }
  } catch (...) {
    return refuse(TSS_ENOSPACE, me, "no host memory for the list");
  }
  return TSS_OK;
}

}  // extern "C"
