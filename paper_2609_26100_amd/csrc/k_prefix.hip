// Attention over the paged KV cache for sequences that share a prefix (gfx950).
//
// softmax(q K^T) V over a group's tokens falls into the shared pages, which all rows of the
// group see whole, and each sequence's own pages: a launch takes both kinds of blocks (of
// window_core.h, whose states (maximum, sum, outputs) say all about a part of the
// tokens), a second joins a row's states.  The blocks of the shared pages hold the rows of
// the whole group beside each other, so that a page is read once for all of them (once
// for every 128 virtual rows, of an fp32 cache for every 16); they need no masks.
//
// Bound by HBM where the own pages weigh most (64 sequences of 32 heads, 300 own tokens behind
// 8000 shared ones, 446 MB: 92 + 5 us, 4.9 TB/s) or a group has few rows (8 sequences of 32
// heads over 8 kv heads behind 16000 tokens, 66 MB: 16 + 4 us); by the blocks' steps, as in
// k_window.hip, where a page serves many rows (64 of 4 heads a kv head behind 32000 tokens:
// 69 + 7 us, 450 TFLOP/s); by two launches and the walk from the group to its pages
// (five loads one behind the other) where all is short (four beams behind 1008 tokens
// 9.0 + 3.9 us).
//
// A row that stands inside the shared pages cuts them down for its group, to the pages
// that every row sees whole; the rest is read through the sequences' own tables.  Every
// workgroup finds that number itself, a lane for each sequence of the group.  Groups of
// unlike sizes get the same splits, as the host knows the largest only: workgroups that
// find nothing end at once, but those of a small group have short walks.
#include "window_core.h"

#include <algorithm>

namespace tss {

namespace {

constexpr int kPrefixThreads = kRowsPages * 64;

// The arguments as the two kinds of blocks see them.
struct SharedPart : PrefixArgs {
  __device__ explicit SharedPart(const PrefixArgs& a) : PrefixArgs(a) {}
};
struct OwnPart : PrefixArgs {
  __device__ explicit OwnPart(const PrefixArgs& a) : PrefixArgs(a) {}
};

__device__ __forceinline__ int group_first(const PrefixArgs& a, int g) {  // first sequence of group g
  return a.group_offsets ? min(max(a.group_offsets[g], 0), a.n_seqs) : g == 0 ? 0 : a.n_seqs;
}
__device__ __forceinline__ int length_of(const PrefixArgs& a, int s) {
  return max(0, min(min(a.lengths[s], a.max_length), a.table_stride * kPage));
}

// A group's sequences, rows and the pages that its blocks take.
struct Group {
  int s0, s1, r0, rows, shared;
};
__device__ __forceinline__ Group make_group(const PrefixArgs& a, int g) {
  Group x;
  x.s0 = group_first(a, g);
  x.s1 = max(x.s0, group_first(a, g + 1));
  x.shared = min(min(max(a.shared[g], 0), a.max_shared), a.table_stride);
  x.r0 = min(max(a.row_offsets[x.s0], 0), a.rows);
  x.rows = min(max(a.row_offsets[x.s1], x.r0), a.rows) - x.r0;
  int seen = x.shared;  // pages that a lane's sequences see whole
  for (int s = x.s0 + (int)(threadIdx.x & 63); s < x.s1; s += 64) {
    const int q0 = min(max(a.row_offsets[s], 0), a.rows), q1 = min(max(a.row_offsets[s + 1], q0), a.rows);
    if (q1 > q0) seen = min(seen, max(0, length_of(a, s) - (q1 - q0) + 1) / kPage);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) seen = min(seen, __shfl_xor(seen, off));
  x.shared = x.rows > a.max_group_rows ? 0 : __builtin_amdgcn_readfirstlane(seen);
  return x;
}
// The pages that sequence s leaves to its group's blocks.
__device__ __forceinline__ int shared_of(const PrefixArgs& a, int s) {
  int g = 0;  // groups that end before s
  for (int i = threadIdx.x & 63; i < a.n_groups; i += 64) g += group_first(a, i + 1) <= s;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) g += __shfl_xor(g, off);
  g = __builtin_amdgcn_readfirstlane(g);
  return g < a.n_groups && group_first(a, g) <= s ? make_group(a, g).shared : 0;
}

// Rows `first` .. of group g and its shared pages.
__device__ __forceinline__ Block make_block(const SharedPart& a, int g, int first, int most) {
  const Group x = make_group(a, g);
  Block b{};
  b.r0 = x.r0;
  b.rows = x.rows;
  b.v0 = first;
  b.n_v = x.shared > 0 ? max(0, min(most, x.rows * a.group - first)) : 0;
  b.lo = b.hi = x.shared * kPage - 1;
  b.window = INT_MAX;
  b.n_pages = x.shared;
  b.table = a.page_table + (size_t)min(x.s0, a.n_seqs - 1) * a.table_stride;
  return b;
}
template <>
struct Row<SharedPart> {
  __device__ Row() {}
  __device__ Row(const SharedPart&, const Block&, int) {}
  __device__ bool sees(const Block&, int) const { return true; }
};
__device__ __forceinline__ Span span_of(const SharedPart&, const Block& b, int, int) { return Span(b, b.lo, b.hi); }

// Rows `first` .. of sequence s and its pages behind the shared ones.
__device__ __forceinline__ Block make_block(const OwnPart& a, int s, int first, int most, int shared) {
  Block b{};
  b.r0 = min(max(a.row_offsets[s], 0), a.rows);
  b.rows = min(max(a.row_offsets[s + 1], b.r0), a.rows) - b.r0;
  b.p0 = length_of(a, s) - b.rows;
  b.window = INT_MAX;
  b.table = a.page_table + (size_t)s * a.table_stride;
  lay_out(b, first, most, min(b.rows, a.max_rows), a.group);
  b.win_page = shared;
  b.n_pages = b.n_v > 0 ? max(0, (b.hi + kPage) / kPage - shared) : 0;
  return b;
}

// How a launch is cut up.  Bodies: 0 blocks of 16 virtual rows whose waves stream pages of
// their own, 1 and 2 blocks of 64 and 128 rows that share each page through LDS.
struct Cut {
  int body, rows, blocks, splits;
};
struct PrefixPlan {
  Cut shared, own;
};

__host__ __device__ constexpr int body_rows(int body) { return body == 0 ? kFewRows : body == 1 ? 64 : 128; }

template <typename T, int HD, int BODY, typename A, typename S>
__device__ __forceinline__ void run_block(const A& a, const Place& w, const Block& b, S& lds, float* part_o,
                                          float* part_ml) {
  if constexpr (BODY == 0)
    few_block<T, HD, kRowsPages>(a, w, b, FewShared{lds.few.o, lds.few.m, lds.few.l}, part_o, part_ml);
  else
    rows_block<HD, BODY>(a, w, b, lds.ring, part_o, part_ml);
}

// grid: the workgroups of the shared pages (head first, then block, split, group), then those
// of the own ones (head, block, split, sequence).  BP, BO: their bodies.
template <typename T, int HD, int BP, int BO>
__global__ __launch_bounds__(kPrefixThreads, 2) void k_prefix(PrefixArgs args, PrefixPlan p, int n_shared, float* part_o,
                                                             float* part_ml) {
  __shared__ __align__(16) union {
    struct {
      float o[kRowsPages][kFewRows][64 + 4], m[kRowsPages][kFewRows], l[kRowsPages][kFewRows];
    } few;
    uint8_t ring[BP || BO ? kRowsRing<HD> : 16];
  } lds;
  const int heads = args.n_heads;
  if ((int)blockIdx.x < n_shared) {
    const SharedPart a(args);
    int i = blockIdx.x;
    Place w{};
    w.head = i % heads;
    i /= heads;
    w.block = i % p.shared.blocks;
    i /= p.shared.blocks;
    w.split = i % p.shared.splits;
    w.item = i / p.shared.splits;
    w.blocks = p.shared.blocks;
    w.splits = p.shared.splits;
    w.parts = true;
    const Block b = make_block(a, w.item, w.block * body_rows(BP), body_rows(BP));
    run_block<T, HD, BP>(a, w, b, lds, part_o, part_ml);
  } else {
    const OwnPart a(args);
    int i = blockIdx.x - n_shared;
    Place w{};
    w.head = i % heads;
    i /= heads;
    w.block = i % p.own.blocks;
    i /= p.own.blocks;
    w.split = i % p.own.splits;
    w.item = i / p.own.splits;
    w.blocks = p.own.blocks;
    w.splits = p.own.splits;
    w.split0 = n_shared ? p.shared.splits : 0;
    w.parts = w.split0 + w.splits > 1;
    const int shared = n_shared ? shared_of(a, w.item) : 0;
    const Block b = make_block(a, w.item, w.block * body_rows(BO), body_rows(BO), shared);
    // no block of shared pages writes these rows' states
    if (shared == 0 && w.split == 0)
      for (int v = threadIdx.x; v < b.n_v * w.split0; v += kPrefixThreads)
        *(float2*)(part_ml + part_slot(a, b, b.v0 + v % b.n_v, w.head, v / b.n_v) * 2) = make_float2(kLowest, 0.f);
    run_block<T, HD, BO>(a, w, b, lds, part_o, part_ml);
  }
}

// Virtual rows, the body and its blocks.
Cut cut_of(bool f16, int64_t v_rows, int most) {
  Cut c;
  // blocks of 128 rows, which read a page half as often, where they hold the rows as well: 64
  // sequences of 4 heads a kv head behind 32000 tokens 65 us, in blocks of 64 80; 160 rows (of
  // which blocks of 128 leave more empty) behind 8000 32 us in either
  const bool wide = most == 2 && (v_rows + 127) / 128 * 2 == (v_rows + 63) / 64;
  c.body = !f16 || v_rows <= kFewRows ? 0 : wide ? 2 : 1;
  c.rows = body_rows(c.body);
  c.blocks = (int)((v_rows + c.rows - 1) / c.rows);
  c.splits = 1;
  return c;
}

PrefixPlan plan(bool f16, int n_heads, int group, int n_seqs, int max_rows, int max_length, int n_groups,
                int max_group_rows, int max_shared) {
  PrefixPlan p;
  p.shared = cut_of(f16, (int64_t)max_group_rows * group, 2);
  p.own = cut_of(f16, (int64_t)max_rows * group, 1);
  const int64_t all = (max_length + kPage - 1) / kPage;
  if (n_groups == 0 || max_group_rows == 0 || max_shared == 0) p.shared.blocks = 0;
  const int64_t shared = p.shared.blocks ? std::min<int64_t>(max_shared, all) : 0;
  const int64_t own = std::max<int64_t>(1, all - shared);
  const int64_t ws = (int64_t)n_heads * n_groups * p.shared.blocks, wo = (int64_t)n_heads * n_seqs * p.own.blocks;
  // Every workgroup about as many pages (a block of 128 rows takes twice as long for one), and
  // as many of them as run at once, two a CU, or a little more than one a CU where their waves
  // stream pages (8 beams of 32 heads behind 4000 tokens: 8 splits 20.6 us, 13 24.0); but no
  // fewer pages than pay for a state (four beams behind 1008 tokens: 4 splits 10.5 us, 2 12.6;
  // 8 of grouped heads behind 4000: 16 to 24 splits 12.4 to 12.9, 32 14.5).
  auto weight = [](const Cut& c) { return c.body == 2 ? 2.0 : 1.0; };
  auto at_once = [](const Cut& c) { return c.body == 0 ? 300 : 512; };
  const double each = ((double)ws * weight(p.shared) * shared + (double)wo * own) / at_once(p.shared);
  auto splits = [&](const Cut& c, int64_t pages, double each) {
    const int least = c.body == 0 ? 16 : 12;
    const int64_t n = (int64_t)((double)pages / std::max<double>(each / weight(c), least) + 0.999);
    return (int)std::max<int64_t>(1, std::min<int64_t>(n, kMaxSplits / 2));
  };
  p.shared.splits = splits(p.shared, shared, each);
  // a bound that covers the longest walk says nothing of how much is shared: the own pages are cut up
  // as if nothing were, and what is shared leaves splits that end at once (without bounds, two
  // sequences of 20000 own tokens of 32 heads over 8 183 -> 43 us, 8 beams of 100 behind 250
  // shared pages 19.4 -> 22.6)
  p.own.splits = shared < all ? splits(p.own, own, each) : splits(p.own, all, (double)wo * all / at_once(p.own));
  return p;
}

int64_t n_shared_of(const PrefixPlan& p, int n_heads, int n_groups) {
  return (int64_t)n_heads * n_groups * p.shared.blocks * p.shared.splits;
}
// States of a row; 1: none, the outputs are written at once.
int states(const PrefixPlan& p) { return (p.shared.blocks ? p.shared.splits : 0) + p.own.splits; }

template <typename T, int HD, int BP, int BO>
void launch_blocks(const PrefixArgs& a, const PrefixPlan& p, float* part_o, float* part_ml, hipStream_t s) {
  const int64_t n = n_shared_of(p, a.n_heads, a.n_groups);
  const int64_t grid = n + (int64_t)a.n_heads * a.n_seqs * p.own.blocks * p.own.splits;
  TSS_LAUNCH((k_prefix<T, HD, BP, BO>), dim3(grid), dim3(kPrefixThreads), 0, s, a, p, (int)n, part_o, part_ml);
}

template <typename T, int HD>
hipError_t launch_typed(const PrefixArgs& a, float* ws, hipStream_t s) {
  const PrefixPlan p = plan(sizeof(T) == 2, a.n_heads, a.group, a.n_seqs, a.max_rows, a.max_length, a.n_groups,
                            a.max_group_rows, a.max_shared);
  const int n = states(p), heads = a.n_heads * a.group;
  float* part_o = ws;
  float* part_ml = ws + (size_t)n * a.rows * heads * HD;
  if constexpr (sizeof(T) == 2) {
    const int bp = p.shared.body, bo = p.own.body;
    if (bo == 0 && bp == 0) launch_blocks<T, HD, 0, 0>(a, p, part_o, part_ml, s);
    if (bo == 0 && bp == 1) launch_blocks<T, HD, 1, 0>(a, p, part_o, part_ml, s);
    if (bo == 0 && bp == 2) launch_blocks<T, HD, 2, 0>(a, p, part_o, part_ml, s);
    if (bo == 1 && bp <= 1) launch_blocks<T, HD, 1, 1>(a, p, part_o, part_ml, s);
    if (bo == 1 && bp == 2) launch_blocks<T, HD, 2, 1>(a, p, part_o, part_ml, s);
  } else {
    launch_blocks<T, HD, 0, 0>(a, p, part_o, part_ml, s);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || n == 1) return e;
  // as behind the windows' kernels, by waves only after blocks of many rows (four beams behind 1008
  // tokens of 32 heads, a call in a graph, 14.4 us by workgroups, 14.7 by waves; 8 behind 4000 24.0
  // and 24.3)
  if constexpr (sizeof(T) == 2)
    if (n <= kWaveSplits && p.shared.body + p.own.body > 0) {
      TSS_LAUNCH((k_window_join_wave<HD, PrefixArgs>), dim3(a.max_rows, a.n_seqs, (heads + 3) / 4), dim3(256), 0, s, a,
                 n, part_o, part_ml);
      return hipGetLastError();
    }
  TSS_LAUNCH((k_window_join<T, HD, PrefixArgs>), dim3(a.max_rows, a.n_seqs, heads), dim3(256), 0, s, a, n, part_o,
             part_ml);
  return hipGetLastError();
}

}  // namespace

bool prefix_fits(int n_heads, int group, int n_seqs, int max_rows, int n_groups, int max_group_rows) {
  // the join's grid, and workgroups of 16 virtual rows in kMaxSplits splits each
  return window_fits(n_heads, group, n_seqs, max_rows) && n_groups <= 65535 &&
         ((int64_t)max_group_rows * group / kFewRows + 1) * n_heads * std::max(n_groups, 1) +
                 ((int64_t)max_rows * group / kFewRows + 1) * n_heads * std::max(n_seqs, 1) <
             (1 << 22);
}

size_t prefix_bytes(bool f16, int head_dim, int n_heads, int group, int n_seqs, int rows, int max_rows, int max_length,
                    int n_groups, int max_group_rows, int max_shared) {
  const int n =
      states(plan(f16, n_heads, group, n_seqs, max_rows, max_length, n_groups, max_group_rows, max_shared));
  return n == 1 ? 0 : (size_t)n * rows * n_heads * group * (head_dim + 2) * 4;
}

hipError_t launch_prefix(bool f16, int head_dim, const PrefixArgs& a, void* workspace, hipStream_t s) {
  float* ws = (float*)workspace;
  if (f16) return head_dim == 128 ? launch_typed<_Float16, 128>(a, ws, s) : launch_typed<_Float16, 64>(a, ws, s);
  return head_dim == 128 ? launch_typed<float, 128>(a, ws, s) : launch_typed<float, 64>(a, ws, s);
}

}  // namespace tss
