// Attention with a sliding window and sinks over the paged KV cache (gfx950).
//
// A row at position p sees token t when t <= p and (t < sinks or t > p - window).
// The query heads that share a kv head are rows beside each other (row i of
// group head j is "virtual" row i * group + j), so that each page is read once
// for all of them.  A workgroup takes a block of virtual rows of one (sequence,
// kv head) and walks only the pages that some row of it sees: those of the
// sinks, then those from the first row's window on.
//
// One pass over the pages with the running maximum and sum of the softmax, in
// powers of two:
//   * S = K Q^T puts tokens on the MFMA rows and query rows on its columns:
//     lane (row r16, group grp) holds the scores of tokens 4 grp .. 4 grp + 3 of a
//     page.  The maximum takes one exchange over the four lanes of a row, the
//     sums are kept per lane and added at the end.
//   * O^T = V^T P^T takes the scores' layout as its second operand without
//     moving them.
// Two kernels: few rows (up to 16) are bound by the cache's bytes, so each wave
// streams pages of its own into registers and the waves' states meet at the end;
// many rows share each page through LDS, a wave for each 16 or 32 rows.  Where
// the blocks are too few for the chip, each block's pages are split among several
// workgroups and a second launch joins their states.  The blocks stand in window_core.h.
//
// Long contexts of few rows are bound by HBM (5 rows of 32 heads over 8 kv heads
// and 100003 tokens, 410 MB: 72 + 5 us, 5.3 TB/s), short ones by their two launches
// (one row of 32 heads over 1028 tokens 8.4 + 3.1 us).  Blocks of many rows take, for
// each step of 64 tokens and 128 rows, 0.43 us each of a SIMD's matrix products and of
// its LDS reads and as much of the softmax, and two waves a SIMD hide little of one
// behind the other (2048 rows of 32 heads, 1028 tokens each: 52 us a call in a loop, 650 TFLOP/s,
// with the loads before the products 57.7; traced 59 and 65).
//
// Of an fp16 cache, the probabilities go to fp16 for the second product (two terms each
// would take twice its instructions): outputs are off by 2.3e-4 to 2.9e-4 of their size
// against 64 bits (root mean square), where the rounding of the result alone is 2.1e-4.
//
// Tokens that no row of the block sees may hold anything: their scores are
// replaced, and their V, which the product would multiply by 0, is cleared.
#include "window_core.h"

#include <algorithm>

namespace tss {

namespace {

// grid (kv head + heads * block, sequence, split)
template <typename T, int HD, typename A>
__global__ __launch_bounds__(kFewWaves * 64, 2) void k_window_few(A a, int splits, float* part_o, float* part_ml) {
  __shared__ float s_o[kFewWaves][kFewRows][64 + 4];
  __shared__ float s_m[kFewWaves][kFewRows], s_l[kFewWaves][kFewRows];
  const FewShared sh{s_o, s_m, s_l};
  const int block = blockIdx.x / a.n_heads;
  const Place w{(int)blockIdx.y, (int)blockIdx.x % a.n_heads, block, (int)gridDim.x / a.n_heads, (int)blockIdx.z,
                splits, 0, splits > 1};
  few_block<T, HD, kFewWaves>(a, w, make_block(a, w.item, block * kFewRows, kFewRows), sh, part_o, part_ml);
}

// grid as k_window_few
template <int HD, int TILES, typename A>
__global__ __launch_bounds__(kRowsPages * 64, 2) void k_window_rows(A a, int splits, int blocks, float* part_o,
                                                                   float* part_ml) {
  constexpr int ROWS = kRowsPages * TILES * 16;
  __shared__ __align__(16) uint8_t ring[kRowsRing<HD>];
  // the last rows first: without a window theirs is the longest walk
  const int block = blocks - 1 - (int)blockIdx.x / a.n_heads;
  const Place w{(int)blockIdx.y, (int)blockIdx.x % a.n_heads, block, blocks, (int)blockIdx.z, splits, 0, splits > 1};
  rows_block<HD, TILES>(a, w, make_block(a, w.item, block * ROWS, ROWS), ring, part_o, part_ml);
}

// How a launch is cut up: virtual rows of a block, blocks of a sequence, splits of
// a block's pages.
struct Plan {
  int rows, blocks, splits;
};
// pages: most that a walk can have; seqs: sequences or items.
Plan plan(bool f16, int n_heads, int64_t v_rows, int64_t seqs, int64_t pages) {
  Plan p;
  // blocks of 64 rows while all of them run at once (two a CU); where there are more,
  // blocks of 128, which read LDS and L2 half as often: 2048 rows behind 2048 tokens
  // in 1024 blocks of 64 69.9 us and in 512 of 128 56.7, 64 sequences of 17 rows of 4
  // heads a kv head 135 and 103, but 777 rows of 4 heads a kv head in 392 of 64 20.5
  // and in 200 of 128 (two splits) 35.9
  const int64_t shorts = n_heads * seqs * ((v_rows + 63) / 64);
  p.rows = !f16 || v_rows <= kFewRows ? kFewRows : v_rows <= 64 || shorts <= 512 ? 64 : 128;
  p.blocks = (int)((v_rows + p.rows - 1) / p.rows);
  const int64_t wgs = n_heads * seqs * p.blocks;
  p.splits = 1;
  if (p.rows == kFewRows) {
    // a wave of few rows takes most of a SIMD's registers: one workgroup a CU.  Splits
    // are worth their second launch where the blocks leave most of the chip idle and
    // each still has some pages to walk: one row over 1028 tokens of 32 heads 15.1 us in
    // one split, 10.8 + 3.6 in two, 8.4 + 3.0 in four
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({kMaxSplits, 256 / wgs, pages / kFewLeast}));
    return p;
  }
  // the time of a step of four pages, of the second launch, and of a (row, head)'s state
  // of a split written and read, in us: 300 rows of 32 heads over 700 tokens take 20.0
  // us in one split and 23.9 in three, over 5000 tokens 121 and 55
  constexpr double kStep = 1.1, kLaunch = 3.0, kState = 0.27e-3;
  const int64_t steps = (pages + kRowsPages - 1) / kRowsPages;
  const int64_t most = std::min<int64_t>({kMaxSplits, 512 / wgs, pages / kRowsLeast});
  double best = kStep * (double)steps;
  for (int64_t n = 2; n <= most; ++n) {
    const double t = kStep * (double)((steps + n - 1) / n) + kLaunch + kState * (double)(n * v_rows * n_heads * seqs);
    if (t >= best) continue;
    best = t;
    p.splits = (int)n;
  }
  return p;
}

template <typename T, int HD, typename A>
void launch_join(const A& a, int rows, int seqs, const Plan& p, const float* part_o, const float* part_ml,
                 hipStream_t s) {
  const int heads = a.n_heads * a.group;
  if constexpr (std::is_same<T, _Float16>::value)
    if (p.rows != kFewRows && p.splits <= kWaveSplits) {
      TSS_LAUNCH((k_window_join_wave<HD, A>), dim3(rows, seqs, (heads + 3) / 4), dim3(256), 0, s, a, p.splits, part_o,
                 part_ml);
      return;
    }
  TSS_LAUNCH((k_window_join<T, HD, A>), dim3(rows, seqs, heads), dim3(256), 0, s, a, p.splits, part_o, part_ml);
}

// Pages that a block of `rows` rows walks at most.
int64_t walk_pages(int64_t rows, int64_t max_length, int64_t sinks, int64_t window) {
  const int64_t all = (max_length + kPage - 1) / kPage;
  return window > 0 ? std::min(all, (sinks + kPage - 1) / kPage + (window + rows + 2 * kPage - 3) / kPage) : all;
}
Plan plan(bool f16, int n_heads, int group, int n_seqs, int max_rows, int max_length, int sinks, int window) {
  Plan p = plan(f16, n_heads, (int64_t)max_rows * group, n_seqs, INT_MAX);
  const int64_t rows = std::min<int64_t>(max_rows, (p.rows + group - 1) / group + 1);
  return plan(f16, n_heads, (int64_t)max_rows * group, n_seqs, walk_pages(rows, max_length, sinks, window));
}

}  // namespace

bool window_fits(int n_heads, int group, int n_seqs, int max_rows) {
  // grids: (heads * blocks, sequences, splits) and (rows, sequences, query heads)
  return n_seqs <= 65535 && (int64_t)n_heads * group <= 65535 &&
         (int64_t)max_rows * group / kFewRows * n_heads < (1 << 22);
}

size_t window_bytes(bool f16, int head_dim, int n_heads, int group, int n_seqs, int rows, int max_rows, int max_length,
                    int sinks, int window) {
  const Plan p = plan(f16, n_heads, group, n_seqs, max_rows, max_length, sinks, window);
  return p.splits == 1 ? 0 : (size_t)p.splits * rows * n_heads * group * (head_dim + 2) * 4;
}

template <typename T, int HD>
static hipError_t launch_typed(const WindowArgs& a, float* ws, hipStream_t s) {
  const Plan p = plan(sizeof(T) == 2, a.n_heads, a.group, a.n_seqs, a.max_rows, a.max_length, a.sinks, a.window);
  float* part_o = ws;
  float* part_ml = ws + (size_t)p.splits * a.rows * a.n_heads * a.group * HD;
  const dim3 grid(a.n_heads * p.blocks, a.n_seqs, p.splits);
  if (p.rows == kFewRows) {
    TSS_LAUNCH((k_window_few<T, HD, WindowArgs>), grid, dim3(kFewWaves * 64), 0, s, a, p.splits, part_o, part_ml);
  } else if constexpr (sizeof(T) == 2) {
    const dim3 block(kRowsPages * 64);
    if (p.rows == 64)
      TSS_LAUNCH((k_window_rows<HD, 1, WindowArgs>), grid, block, 0, s, a, p.splits, p.blocks, part_o, part_ml);
    else
      TSS_LAUNCH((k_window_rows<HD, 2, WindowArgs>), grid, block, 0, s, a, p.splits, p.blocks, part_o, part_ml);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  launch_join<T, HD>(a, a.max_rows, a.n_seqs, p, part_o, part_ml, s);
  return hipGetLastError();
}

hipError_t launch_window(bool f16, int head_dim, const WindowArgs& a, void* workspace, hipStream_t s) {
  float* ws = (float*)workspace;
  if (f16) return head_dim == 128 ? launch_typed<_Float16, 128>(a, ws, s) : launch_typed<_Float16, 64>(a, ws, s);
  return head_dim == 128 ? launch_typed<float, 128>(a, ws, s) : launch_typed<float, 64>(a, ws, s);
}

template <int HD>
static hipError_t launch_pass_typed(const WindowPassArgs& a, hipStream_t s) {
  // blocks as a call's, without splits, and as many as the report of a launch has items for
  // (1000 rows of 32 heads under 512 + 4 tokens 16.5 us in blocks of 64, 20.0 in blocks of 128)
  const bool shorts = (int64_t)a.n_heads * ((a.rows + 63) / 64) <= 512 && a.rows <= 64 * kAttnMaxItems;
  const int blocks = shorts ? (a.rows + 63) / 64 : (a.rows + 127) / 128;
  const dim3 grid(a.n_heads * blocks, 1, 1), block(kRowsPages * 64);
  float* none = nullptr;
  if (shorts)
    TSS_LAUNCH((k_window_rows<HD, 1, WindowPassArgs>), grid, block, 0, s, a, 1, blocks, none, none);
  else
    TSS_LAUNCH((k_window_rows<HD, 2, WindowPassArgs>), grid, block, 0, s, a, 1, blocks, none, none);
  return hipGetLastError();
}

static_assert(kPromptRows <= 128 * kAttnMaxItems, "a block each in the report");
hipError_t launch_window_pass(int head_dim, const WindowPassArgs& a, hipStream_t s) {
  if (a.rows < 1 || a.rows > kPromptRows) return hipErrorInvalidValue;
  return head_dim == 128 ? launch_pass_typed<128>(a, s) : launch_pass_typed<64>(a, s);
}

template <typename T, int HD>
static hipError_t launch_step_typed(int n_items, const WindowStepArgs& a, float* part_o, float* part_ml,
                                    size_t part_slots, hipStream_t s) {
  int64_t rows = 0, pages = 0;
  for (int i = 0; i < n_items; ++i) {
    const WindowStepArgs::Item& it = a.item[i];
    rows = std::max<int64_t>(rows, it.rows);
    // rows at the context's end and draft slots behind it
    pages = std::max(pages, walk_pages(it.slots, a.max_length, it.sinks, it.window == INT_MAX ? 0 : it.window));
  }
  Plan p = plan(sizeof(T) == 2, a.n_heads, rows, n_items, pages);
  if (p.rows > 64) return hipErrorInvalidValue;  // items have at most 64 rows
  // a slot holds 64 rows of one head
  p.splits = (int)std::min<int64_t>(p.splits, std::max<int64_t>(1, part_slots * 64 / ((int64_t)a.rows * a.n_heads)));
  const dim3 grid(a.n_heads * p.blocks, n_items, p.splits);
  if (p.rows == kFewRows)
    TSS_LAUNCH((k_window_few<T, HD, WindowStepArgs>), grid, dim3(kFewWaves * 64), 0, s, a, p.splits, part_o, part_ml);
  else if constexpr (sizeof(T) == 2)
    TSS_LAUNCH((k_window_rows<HD, 1, WindowStepArgs>), grid, dim3(kRowsPages * 64), 0, s, a, p.splits, p.blocks, part_o, part_ml);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.splits == 1) return e;
  // the timing of a launch is that of the one above
  const LaunchTiming timing = launch_timing();
  launch_timing() = LaunchTiming{};
  launch_join<T, HD>(a, (int)rows, n_items, p, part_o, part_ml, s);
  launch_timing() = timing;
  return hipGetLastError();
}

hipError_t launch_window_step(bool f16, int head_dim, int n_items, const WindowStepArgs& a, float* part_o,
                              float* part_ml, size_t part_slots, hipStream_t s) {
  if (n_items < 1 || n_items > kAttnMaxItems) return hipErrorInvalidValue;
  if (f16)
    return head_dim == 128 ? launch_step_typed<_Float16, 128>(n_items, a, part_o, part_ml, part_slots, s)
                           : launch_step_typed<_Float16, 64>(n_items, a, part_o, part_ml, part_slots, s);
  return head_dim == 128 ? launch_step_typed<float, 128>(n_items, a, part_o, part_ml, part_slots, s)
                         : launch_step_typed<float, 64>(n_items, a, part_o, part_ml, part_slots, s);
}

}  // namespace tss
