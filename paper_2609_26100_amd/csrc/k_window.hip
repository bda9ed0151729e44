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
// workgroups and a second launch joins their states.
//
// Long contexts of few rows are bound by HBM (5 rows of 32 heads over 8 kv heads
// and 100003 tokens, 410 MB: 74 + 5 us, 5.2 TB/s), short ones by their two launches
// (one row of 32 heads over 1028 tokens 8.9 + 3.1 us).  Blocks of many rows take, for
// each step of 64 tokens and 128 rows, 0.43 us each of a SIMD's matrix products and of
// its LDS reads and as much of the softmax, and two waves a SIMD hide little of one
// behind the other (2048 rows of 32 heads, 1028 tokens each: 57 us, 600 TFLOP/s).
//
// Of an fp16 cache, the probabilities go to fp16 for the second product (two terms each
// would take twice its instructions): outputs are off by 2.3e-4 to 2.9e-4 of their size
// against 64 bits (root mean square), where the rounding of the result alone is 2.1e-4.
//
// Tokens that no row of the block sees may hold anything: their scores are
// replaced, and their V, which the product would multiply by 0, is cleared.
#include "../../include/tss.h"
#include "tss_internal.h"

#include <algorithm>
#include <climits>
#include <type_traits>

namespace tss {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxSplits = 64;
// Pages that a split has at least: two steps of four pages for the kernel of many
// rows (33 rows over 500 tokens of 32 heads 11.0 us, with sixteen 13.2), two for each
// of eight waves for that of few.
constexpr int kFewLeast = 16, kRowsLeast = 8;
constexpr float kLowest = -3e38f;  // running maximum of a row that has seen nothing
// A row's reference is raised where a score exceeds the maximum that set it by this
// (in powers of two): larger probabilities fit fp16 as well (their rounding is
// relative), and almost no step has to rescale its outputs, where with a threshold of
// 0 some row of sixteen nearly always rises.
constexpr float kRise = 8.f;
// Probabilities that go to fp16 are relative to a reference this many powers of two
// below the maximum, so that the largest is 2^15 in the kernel of few rows and, with
// kRise, 2^7 to 2^15 in that of many.  A small one's rounding is then at most 2^-40 or
// 2^-32 of the largest; with the maximum as the reference it would be 2^-25, and 20000
// tokens of 2^-26 each, 3e-4 of a row's weight together, would come to nothing.  The
// sums have the same factor, so it cancels.
constexpr float kFewDown = 15.f, kRowsDown = 7.f;
// A probability is 2^(S scale - m) in one fma, whose product is not rounded while m
// was: up to kFar that makes a factor of at most 2^(2^-8) that the sums share, at 1e9 one
// of up to 2^32, beyond fp16.  Where a reference maximum is farther from zero the
// product is rounded first (the test and kRowsDown: 57.6 -> 58.0 us for 2048 rows of 32
// heads, 53.9 -> 54.1 for 300 over 5000 tokens).
constexpr float kFar = 65536.f;

// Over the four lanes l, l ^ 16, l ^ 32, l ^ 48 of a row.
__device__ __forceinline__ float max4(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float sum4(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(h[0]) + __uint_as_float(h[1]);
}

// S scale - m with the product rounded by itself (the empty asm keeps it out of an fma).
__device__ __forceinline__ void round_exponents(f32x4& S, float scale, float m) {
#pragma unroll
  for (int v = 0; v < 4; ++v) {
    float x = S[v] * scale;
    asm volatile("" : "+v"(x));
    S[v] = x - m;
  }
}

// A block of virtual rows of one sequence and the pages it walks.
struct Block {
  int r0, rows;          // first row of the sequence, its rows
  int v0, n_v;           // first virtual row of the block, how many it has (0: nothing to do)
  int p0;                // position of the sequence's first row (may be negative: more rows than tokens)
  int lo, hi;            // positions of the block's first and last row, at least -1 (a step: lowest
                         // position of a row, last slot that one sees)
  int n_kv;              // a step's committed context
  int sinks, window;
  int sink_pages, win_page, n_pages;  // page i of the walk: i < sink_pages ? i : win_page + i - sink_pages
  const int32_t* table;

  __device__ int page(int i) const { return i < sink_pages ? i : win_page + (i - sink_pages); }
  // position of a virtual row
  __device__ int pos(int v, int group) const { return max(p0 + v / group, -1); }
  __device__ bool sees(int t, int p) const { return (t <= p) & ((t < sinks) | (t > p - window)); }
  // the walk's place of a page from win_page on
  __device__ int place(int page) const { return page - win_page + sink_pages; }
  // some row of the block sees the token
  __device__ bool live(int t) const { return (t <= hi) & ((t < sinks) | (t > lo - window)); }
};

// Cuts the block out of rows at positions b.p0 on and lays out its walk.
__device__ __forceinline__ void lay_out(Block& b, int first, int most, int n_rows, int group) {
  b.v0 = first;
  b.n_v = max(0, min(most, n_rows * group - first));
  if (b.n_v == 0) return;
  b.lo = b.pos(first, group);
  b.hi = b.pos(first + b.n_v - 1, group);
}
__device__ __forceinline__ void lay_walk(Block& b) {
  if (b.n_v == 0 || b.hi < 0) return;  // no page
  b.win_page = max(0, max(b.lo, 0) - b.window + 1) / kPage;
  b.sink_pages = min((b.sinks + kPage - 1) / kPage, b.win_page);
  b.n_pages = b.sink_pages + b.hi / kPage - b.win_page + 1;
}

// Block `first` .. of sequence s of a call.
__device__ __forceinline__ Block make_block(const WindowArgs& a, int s, int first, int most) {
  Block b{};
  b.r0 = min(max(a.row_offsets[s], 0), a.rows);
  b.rows = min(max(a.row_offsets[s + 1], b.r0), a.rows) - b.r0;
  const int len = max(0, min(min(a.lengths[s], a.max_length), a.table_stride * kPage));
  b.p0 = len - b.rows;
  b.sinks = a.sinks;
  b.window = a.window > 0 ? a.window : INT_MAX;
  b.table = a.page_table + (size_t)s * a.table_stride;
  lay_out(b, first, most, min(b.rows, a.max_rows), a.group);
  lay_walk(b);
  return b;
}
// Of a prefill pass.
__device__ __forceinline__ Block make_block(const WindowPassArgs& a, int, int first, int most) {
  Block b{};
  b.rows = a.rows;
  b.p0 = a.max_length - a.rows;
  b.sinks = a.sinks;
  b.window = a.window;
  b.table = a.page_table;
  lay_out(b, first, most, a.rows, 1);
  lay_walk(b);
  return b;
}
// Of item s of a step: its rows sit at and behind the end of the context, and see
// draft slots behind it.
__device__ __forceinline__ Block make_block(const WindowStepArgs& a, int s, int first, int most) {
  const WindowStepArgs::Item it = a.item[s];
  Block b{};
  b.r0 = it.row0;
  b.rows = it.rows;
  b.v0 = first;
  b.n_v = max(0, min(most, it.rows - first));
  b.n_kv = a.sp->seq_nkv[it.seg];
  b.sinks = it.sinks;
  b.window = it.window;
  b.table = a.page_table + a.pt_off[it.seg];
  b.lo = b.n_kv;
  b.hi = b.n_kv + it.slots - 1;
  lay_walk(b);
  return b;
}

// What a row sees.  In a step: of the context by its position, of the draft slots
// itself and its ancestors (a window is at least as deep as a tree).
template <typename A>
struct Row {
  int pos;
  __device__ Row() {}
  __device__ Row(const A& a, const Block& b, int v) : pos(b.pos(v, a.group)) {}
  __device__ bool sees(const Block& b, int t) const { return b.sees(t, pos); }
};
template <>
struct Row<WindowStepArgs> {
  int pos, node0;
  uint64_t anc;
  __device__ Row() {}
  __device__ Row(const WindowStepArgs& a, const Block& b, int v) {
    const int r = b.r0 + v;
    pos = b.n_kv + a.sp->depth[r];
    node0 = b.n_kv + a.sp->row_slot0[r];
    anc = a.sp->anc[r];
  }
  __device__ bool sees(const Block& b, int t) const {
    const unsigned j = (unsigned)(t - node0);
    return ((t < b.n_kv) & b.sees(t, pos)) | ((t >= b.n_kv) & (j < 64u) & (bool)((anc >> (j & 63u)) & 1ull));
  }
};

// Places of a walk whose pages' tokens rows of positions a to b (at least -1) all
// have in their windows.  Pages of sinks come besides: the walk begins with them,
// so that page i of the sequence is at place i.
struct Span {
  int all_first, all_last;
  __device__ Span(const Block& w, int a, int b) {
    all_first = w.place(b - w.window < 0 ? 0 : (b - w.window) / kPage + 1);
    all_last = w.place((a + 1) / kPage - 1);
  }
};

// The span of virtual rows v .. w of a block.
__device__ __forceinline__ Span span_of(const WindowArgs& a, const Block& b, int v, int w) {
  return Span(b, b.pos(v, a.group), b.pos(w, a.group));
}
__device__ __forceinline__ Span span_of(const WindowStepArgs&, const Block& b, int, int) {
  return Span(b, b.n_kv - 1, b.n_kv + kMaxNodes - 1);
}

// 16 bytes of a virtual row's query: from dimension 32 c + 8 grp on (fp16), 16 c + 4 grp (fp32).
template <typename T, int HD>
__device__ __forceinline__ uint4 load_q(const WindowArgs& a, const Block& b, int v, int head, int c, int grp) {
  const T* q = (const T*)a.q + (size_t)(b.r0 + v / a.group) * a.q_stride + (size_t)(head * a.group + v % a.group) * HD;
  return *(const uint4*)((const uint8_t*)q + c * 64 + grp * 16);
}
// The verifier's queries are fp32; fp16 modes round them to the products' operands here.
template <typename T, int HD>
__device__ __forceinline__ uint4 load_q_f32(const WindowArgs& a, const Block& b, int v, int head, int c, int grp) {
  const float* q = (const float*)a.q + (size_t)(b.r0 + v) * a.q_stride + (size_t)head * HD;
  if constexpr (sizeof(T) == 4) {
    return *(const uint4*)(q + c * 16 + grp * 4);
  } else {
    const float4 x = *(const float4*)(q + c * 32 + grp * 8), y = *(const float4*)(q + c * 32 + grp * 8 + 4);
    return __builtin_bit_cast(uint4, f16x8{(_Float16)x.x, (_Float16)x.y, (_Float16)x.z, (_Float16)x.w, (_Float16)y.x,
                                           (_Float16)y.y, (_Float16)y.z, (_Float16)y.w});
  }
}
template <typename T, int HD>
__device__ __forceinline__ uint4 load_q(const WindowPassArgs& a, const Block& b, int v, int head, int c, int grp) {
  return load_q_f32<T, HD>(a, b, v, head, c, grp);
}
template <typename T, int HD>
__device__ __forceinline__ uint4 load_q(const WindowStepArgs& a, const Block& b, int v, int head, int c, int grp) {
  return load_q_f32<T, HD>(a, b, v, head, c, grp);
}

// Where dimension d of a row and query head is stored; dimensions d .. d + 7 (d a multiple
// of 8, fp16) stand together.
template <typename T, int HD>
__device__ __forceinline__ T* out_at(const WindowArgs& a, int row, int qh, int d) {
  return (T*)a.o + (size_t)row * a.o_stride + (size_t)qh * HD + d;
}
template <typename T, int HD>
__device__ __forceinline__ T* out_at(const WindowPassArgs& a, int row, int qh, int d) {
  return (T*)a.o + act_index<T>(row, qh * HD + d, a.n_heads * HD);
}
template <typename T, int HD>
__device__ __forceinline__ T* out_at(const WindowStepArgs& a, int row, int qh, int d) {
  return (T*)a.o + act_index<T>(row, qh * HD + d, a.n_heads * HD);
}

// The split that a launch took, for inspection.
__device__ __forceinline__ void report(const WindowArgs&, const Block&, int, int, int, int) {}
__device__ __forceinline__ void report(const WindowPassArgs& a, const Block& b, int, int block, int blocks, int) {
  a.split_out[block] = 1;
  a.split_out[kAttnMaxItems + block] = b.n_v;
  if (block == 0) a.split_out[2 * kAttnMaxItems] = blocks;
}
__device__ __forceinline__ void report(const WindowStepArgs& a, const Block& b, int item, int block, int, int splits) {
  if (block > 0) return;
  a.split_out[item] = splits;
  a.split_out[kAttnMaxItems + item] = b.rows;
  if (item == 0) a.split_out[2 * kAttnMaxItems] = gridDim.y;
}

// Words of a lane's V piece (tokens 0, 1 and 2, 3 of its group) that are kept.
__device__ __forceinline__ uint2 keep16(const Block& b, int t, bool there) {
  auto half = [&](int u) { return (there & b.live(t + u)) ? 0xffffu : 0u; };
  return uint2{half(0) | half(1) << 16, half(2) | half(3) << 16};
}

__device__ __forceinline__ uint4 both(uint4 a, uint4 b) { return uint4{a.x & b.x, a.y & b.y, a.z & b.z, a.w & b.w}; }

template <typename T, int HD>
__device__ __forceinline__ const uint8_t* page_k(const WindowArgs& a, int id, int head) {
  return a.kv_pages + ((size_t)id * 2 * a.n_heads + head) * (kPage * HD * sizeof(T));
}

// slot of a virtual row's partial state
__device__ __forceinline__ size_t part_slot(const WindowArgs& a, const Block& b, int v, int head, int split) {
  return ((size_t)split * a.rows + b.r0 + v / a.group) * (a.n_heads * a.group) + head * a.group + v % a.group;
}

// Steps of a split: an equal share, but no fewer than `least`.
__device__ __forceinline__ int split_steps(int steps, int splits, int least) {
  return max(least, (steps + splits - 1) / splits);
}

// --- up to 16 virtual rows ------------------------------------------------------

constexpr int kFewWaves = 8, kFewRows = 16;

// A page in a wave's registers.  Lane (r16, grp): piece c of K holds 16 bytes of
// token r16 from byte 64 c + 16 grp on; piece i of V holds tokens 4 grp .. + 3 of two
// (fp16: 32 i + 2 r16, + 1) or one (fp32: 16 i + r16) dimensions.
template <typename T, int HD>
struct Page {
  static constexpr int N = HD * (int)sizeof(T) / 64;
  uint4 k[N], v[N];
  int i, number;  // place in the walk, page of the sequence (scalars)
  bool there;     // its id is one of the pool's

  __device__ __forceinline__ void load(const WindowArgs& a, int place, int page, int id, int head, int r16, int grp) {
    i = place;
    number = page;
    there = (unsigned)id < (unsigned)a.n_pages;
    const uint8_t* kb = page_k<T, HD>(a, there ? id : 0, head);
    const uint8_t* vb = kb + (size_t)a.n_heads * (kPage * HD * sizeof(T));
#pragma unroll
    for (int c = 0; c < N; ++c) k[c] = *(const uint4*)(kb + (unsigned)(r16 * HD * (int)sizeof(T) + grp * 16 + c * 64));
#pragma unroll
    for (int c = 0; c < N; ++c) v[c] = *(const uint4*)(vb + (unsigned)(grp * HD * 4 * (int)sizeof(T) + r16 * 16 + c * 256));
  }
};

template <typename T, int HD>
__device__ __forceinline__ f32x4 scores(const Page<T, HD>& pg, const uint4* q) {
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < Page<T, HD>::N; ++c) {
    if constexpr (sizeof(T) == 2) {
      s = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, pg.k[c]), __builtin_bit_cast(f16x8, q[c]), s,
                                                 0, 0, 0);
    } else {
      const f32x4 x = __builtin_bit_cast(f32x4, pg.k[c]), y = __builtin_bit_cast(f32x4, q[c]);
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], s, 0, 0, 0);
    }
  }
  return s;
}

// Outputs of a lane: o[n][v] is dimension dim_of(n, v) of row r16.
template <typename T>
__device__ __forceinline__ int dim_of(int n, int v, int grp) {
  if constexpr (sizeof(T) == 2) return 32 * (n >> 1) + 8 * grp + 2 * v + (n & 1);
  return 16 * n + 4 * grp + v;
}

// grid (kv head + heads * block, sequence, split)
template <typename T, int HD, typename A>
__global__ __launch_bounds__(kFewWaves * 64, 2) void k_window_few(A a, int splits, float* part_o, float* part_ml) {
  constexpr int PP = sizeof(T) == 2 ? 2 : 1;  // pages of a step
  constexpr int N = Page<T, HD>::N, NO = HD / 16;
  constexpr int LD = 64 + 4;
  __shared__ float s_o[kFewWaves][kFewRows][LD];
  __shared__ float s_m[kFewWaves][kFewRows], s_l[kFewWaves][kFewRows];
  const int head = blockIdx.x % a.n_heads;
  const Block b = make_block(a, blockIdx.y, blockIdx.x / a.n_heads * kFewRows, kFewRows);
  if (b.n_v == 0) return;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int r16 = lane & 15, grp = lane >> 4;
  const int vrow = b.v0 + min(r16, b.n_v - 1);     // lanes past the block's rows do the last one again
  const Row<A> row(a, b, vrow);
  const Span span = span_of(a, b, b.v0, b.v0 + b.n_v - 1);
  const int full_sinks = b.sinks / kPage;

  // this split's pages, from `from`; wave w takes steps w, w + 8, ...
  const int steps = (b.n_pages + PP - 1) / PP, per = split_steps(steps, splits, kFewLeast / PP);
  const int st0 = blockIdx.z * per, n_st = min(per, steps - st0);
  if (head == 0 && blockIdx.z == 0 && tid == 0)
    report(a, b, blockIdx.y, blockIdx.x / a.n_heads, gridDim.x / a.n_heads, max(1, (steps + per - 1) / per));
  if (n_st <= 0 && blockIdx.z > 0) {  // nothing left for this split
    if (tid < b.n_v) *(float2*)(part_ml + part_slot(a, b, b.v0 + tid, head, blockIdx.z) * 2) = make_float2(kLowest, 0.f);
    return;
  }
  int ids = 0;
  auto walk = [&](int st, int p) { return (st0 + st) * PP + p; };  // page p of this split's step st
  auto load_ids = [&](int st) {  // of this wave's 64 / PP steps from st on
    const int i = walk(st + lane / PP * kFewWaves, lane % PP);
    ids = b.table[b.page(min(i, b.n_pages - 1))];
  };
  uint4 q[N];
#pragma unroll
  for (int c = 0; c < N; ++c) q[c] = load_q<T, HD>(a, b, vrow, head, c, grp);
  f32x4 o[NO];
#pragma unroll
  for (int n = 0; n < NO; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kLowest, l = 0.f;

  Page<T, HD> buf[2][PP];
  auto fetch = [&](Page<T, HD>* pg, int st) {
    if (((st - wave) / kFewWaves) % (64 / PP) == 0) load_ids(st);
    const int j = ((st - wave) / kFewWaves) % (64 / PP) * PP;
#pragma unroll
    for (int p = 0; p < PP; ++p) {
      const int i = walk(st, p);
      const int id = __builtin_amdgcn_readlane(ids, j + p);
      pg[p].load(a, i, b.page(min(i, b.n_pages - 1)), i < b.n_pages ? id : -1, head, r16, grp);
    }
  };
  auto compute = [&](Page<T, HD>* pg) {
    f32x4 S[PP];
    bool whole = true;
#pragma unroll
    for (int p = 0; p < PP; ++p) {
      S[p] = scores<T, HD>(pg[p], q);
      if (!pg[p].there || pg[p].i > span.all_last || (pg[p].i >= full_sinks && pg[p].i < span.all_first)) {
        whole = false;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const bool seen = pg[p].there & row.sees(b, pg[p].number * kPage + 4 * grp + v);
          S[p][v] = seen ? S[p][v] : -INFINITY;
        }
      }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int p = 0; p < PP; ++p)
#pragma unroll
      for (int v = 0; v < 4; ++v) mx = fmaxf(mx, S[p][v]);
    mx *= a.scale_log2;
    if constexpr (sizeof(T) == 2) mx -= fabsf(mx) > kFar ? 0.f : kFewDown;
    mx = max4(fmaxf(m, mx));
    const float alpha = __builtin_amdgcn_exp2f(m - mx);
    m = mx;
    if (__any(fabsf(m) > kFar)) {
#pragma unroll
      for (int p = 0; p < PP; ++p) round_exponents(S[p], a.scale_log2, m);
    } else {
#pragma unroll
      for (int p = 0; p < PP; ++p)
#pragma unroll
        for (int v = 0; v < 4; ++v) S[p][v] = S[p][v] * a.scale_log2 - m;
    }
    float sum = 0.f;
#pragma unroll
    for (int p = 0; p < PP; ++p)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        S[p][v] = __builtin_amdgcn_exp2f(S[p][v]);
        sum += S[p][v];
      }
    l = l * alpha + sum;
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int n = 0; n < NO; ++n) o[n] *= alpha;
    }
    if (!whole) {
#pragma unroll
      for (int p = 0; p < PP; ++p) {
        const int t = pg[p].number * kPage + 4 * grp;
        if constexpr (sizeof(T) == 2) {
          const uint2 k = keep16(b, t, pg[p].there);
#pragma unroll
          for (int i = 0; i < N; ++i) pg[p].v[i] = both(pg[p].v[i], uint4{k.x, k.y, k.x, k.y});
        } else {
          auto word = [&](int u) { return (pg[p].there & b.live(t + u)) ? ~0u : 0u; };
          const uint4 k = {word(0), word(1), word(2), word(3)};
#pragma unroll
          for (int i = 0; i < N; ++i) pg[p].v[i] = both(pg[p].v[i], k);
        }
      }
    }
    if constexpr (sizeof(T) == 2) {
      // k = 8 grp + 4 p + u is token 4 grp + u of page p
      f16x8 P;
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int v = 0; v < 4; ++v) P[4 * p + v] = (_Float16)S[p][v];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const uint4 va = pg[0].v[i], vb = pg[PP - 1].v[i];
        o[2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, uint4{va.x, va.y, vb.x, vb.y}), P,
                                                          o[2 * i], 0, 0, 0);
        o[2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, uint4{va.z, va.w, vb.z, vb.w}),
                                                              P, o[2 * i + 1], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const f32x4 x = __builtin_bit_cast(f32x4, pg[0].v[i]);
#pragma unroll
        for (int v = 0; v < 4; ++v) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[v], S[0][v], o[i], 0, 0, 0);
      }
    }
  };

  if (wave < n_st) {
    fetch(buf[0], wave);
    for (int st = wave; st < n_st; st += 2 * kFewWaves) {
      if (st + kFewWaves < n_st) fetch(buf[1], st + kFewWaves);
      compute(buf[0]);
      if (st + kFewWaves >= n_st) break;
      if (st + 2 * kFewWaves < n_st) fetch(buf[0], st + 2 * kFewWaves);
      compute(buf[1]);
    }
  }

  // the waves' states meet, 64 dimensions at a time
  l = sum4(l);
  if (grp == 0) {
    s_m[wave][r16] = m;
    s_l[wave][r16] = l;
  }
  const int orow = tid >> 5, od = (tid & 31) * 2;  // a thread's two outputs of a round
#pragma unroll
  for (int h = 0; h < HD / 64; ++h) {
    if (h) __syncthreads();
#pragma unroll
    for (int n = 4 * h; n < 4 * h + 4; ++n)
#pragma unroll
      for (int v = 0; v < 4; ++v) s_o[wave][r16][dim_of<T>(n, v, grp) - 64 * h] = o[n][v];
    __syncthreads();
    float top = kLowest;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, s_m[w][orow]);
    float L = 0.f, x = 0.f, y = 0.f;
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w][orow] - top);
      const float2 p = *(const float2*)&s_o[w][orow][od];
      L += f * s_l[w][orow];
      x += f * p.x;
      y += f * p.y;
    }
    if (orow < b.n_v) {
      const int v = b.v0 + orow;
      if (splits > 1) {
        const size_t slot = part_slot(a, b, v, head, blockIdx.z);
        *(float2*)(part_o + slot * HD + 64 * h + od) = make_float2(x, y);
        if (h == 0 && od == 0) *(float2*)(part_ml + slot * 2) = make_float2(top, L);
      } else {
        const float inv = L > 0.f ? 1.f / L : L;  // 0 for a row that sees nothing, NaN stays
        T* to = out_at<T, HD>(a, b.r0 + v / a.group, head * a.group + v % a.group, 64 * h + od);
        to[0] = (T)(x * inv);
        to[1] = (T)(y * inv);
      }
    }
  }
}

// --- many rows (fp16) --------------------------------------------------------------

constexpr int kRowsPages = 4, kRowsStages = 2;

// Four waves of TILES 16-row tiles walk the pages together, four pages a step, one
// loaded by each wave into an LDS ring by global -> LDS loads, two steps in flight.
// K chunk c covers dims 32 c .. + 31 (16 tokens x 64 bytes of a page), V chunk i
// dims 32 i .. + 31 of four token groups (4 x 256 bytes): each is one KiB load, read
// back lane by lane in order.  grid as k_window_few.
template <int HD, int TILES, typename A>
__global__ __launch_bounds__(kRowsPages * 64, 2) void k_window_rows(A a, int splits, int blocks, float* part_o,
                                                                   float* part_ml) {
  constexpr int NK = HD / 32;              // KiB of a K (or V) page block
  constexpr int STAGE = kRowsPages * 2 * NK * 1024;
  constexpr int ROWS = kRowsPages * TILES * 16;
  __shared__ __align__(16) uint8_t ring[kRowsStages * STAGE];
  const int head = blockIdx.x % a.n_heads;
  // the last rows first: without a window theirs is the longest walk
  const int block = blocks - 1 - (int)blockIdx.x / a.n_heads;
  const Block b = make_block(a, blockIdx.y, block * ROWS, ROWS);
  if (b.n_v == 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int r16 = lane & 15, grp = lane >> 4;
  const int steps = (b.n_pages + kRowsPages - 1) / kRowsPages;
  const int per = split_steps(steps, splits, kRowsLeast / kRowsPages);
  const int st0 = blockIdx.z * per, n_st = max(0, min(per, steps - st0));
  if (head == 0 && blockIdx.z == 0 && threadIdx.x == 0)
    report(a, b, blockIdx.y, block, blocks, max(1, (steps + per - 1) / per));
  if (n_st == 0 && blockIdx.z > 0) {  // nothing left for this split
    for (int i = threadIdx.x; i < b.n_v; i += kRowsPages * 64)
      *(float2*)(part_ml + part_slot(a, b, b.v0 + i, head, blockIdx.z) * 2) = make_float2(kLowest, 0.f);
    return;
  }
  const int w0 = wave * TILES * 16;                         // the wave's first row of the block
  const bool on = w0 < b.n_v;
  const Span span = span_of(a, b, b.v0 + w0, b.v0 + min(w0 + TILES * 16, b.n_v) - 1);
  // pages that the sinks fill, and pages of whose tokens each is seen by some row
  // of the block: its first row's from the window's start, its last row's to the end
  const int full_sinks = b.sinks / kPage;
  const int live_first = b.place(b.lo - b.window < 0 ? 0 : (b.lo - b.window) / kPage + 1);
  const int live_last = b.place((b.hi + 1) / kPage - 1);

  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) void*)ring;
  const unsigned koff = (unsigned)(r16 * HD * 2 + grp * 16);          // + c * 64
  const unsigned voff = (unsigned)(grp * HD * 8 + r16 * 16);          // + i * 256
  int ids = 0;  // lane l: id of page l of sixteen steps
  uint64_t good = 0;  // bit l: it is a page of the walk and of the pool
  auto load_ids = [&](int st) {
    const int i = (st0 + st) * kRowsPages + lane;
    const int id = b.table[b.page(min(i, b.n_pages - 1))];
    const bool there = i < b.n_pages && (unsigned)id < (unsigned)a.n_pages;
    good = __ballot(there);
    ids = there ? id : 0;
  };
  auto issue = [&](int st) {
    const int phys = __builtin_amdgcn_readlane(ids, (st * kRowsPages + wave) & 63);
    const uint8_t* kb = page_k<_Float16, HD>(a, phys, head);
    const uint8_t* vb = kb + (size_t)a.n_heads * (kPage * HD * 2);
    const unsigned dst = lds0 + (unsigned)((st % kRowsStages) * STAGE + wave * 2 * NK * 1024);
#pragma unroll
    for (int c = 0; c < NK; ++c) dma_kib(kb, koff + c * 64u, dst + c * 1024u);
#pragma unroll
    for (int c = 0; c < NK; ++c) dma_kib(vb, voff + c * 256u, dst + (NK + c) * 1024u);
  };

  f16x8 q[TILES][NK];
  Row<A> row[TILES];
  f32x4 O[TILES][2 * NK];  // [2 i + j]: dims 32 i + 8 grp + 2 v + j
  float m_run[TILES], l_run[TILES];
  float rise = kRise + kRowsDown;  // scores beyond a reference by more raise it
#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int v = b.v0 + min(w0 + t * 16 + r16, b.n_v - 1);
    row[t] = Row<A>(a, b, v);
#pragma unroll
    for (int c = 0; c < NK; ++c) q[t][c] = __builtin_bit_cast(f16x8, load_q<_Float16, HD>(a, b, v, head, c, grp));
    m_run[t] = kLowest;
    l_run[t] = 0.f;
#pragma unroll
    for (int n = 0; n < 2 * NK; ++n) O[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  if (n_st > 0) {
    load_ids(0);
    issue(0);
  }
  unsigned there = 0;  // bit p: page p of the step is one of the walk's and the pool's
  auto arrive = [&](int st) {
    there = (unsigned)(good >> ((st * kRowsPages) & 63)) & ((1u << kRowsPages) - 1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // every wave's page of step st has landed, and step st - 1 has been read
    asm volatile("" ::: "memory");
    if (st + 1 < n_st) {
      if (((st + 1) & 15) == 0) load_ids(st + 1);
      issue(st + 1);
    }
  };
  // Step st.  EDGE: some of its tokens are seen by no row of the block.
  auto step = [&](int st, auto edge) {
    constexpr bool EDGE = decltype(edge)::value;
    const uint8_t* base = ring + (st % kRowsStages) * STAGE + lane * 16;
    const int i0 = (st0 + st) * kRowsPages, i1 = i0 + kRowsPages - 1;
    f16x8 P[TILES][2];
    f32x4 S[TILES][kRowsPages];
#pragma unroll
    for (int p = 0; p < kRowsPages; ++p) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) S[t][p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        const f16x8 k = *(const f16x8*)(base + (p * 2 * NK + c) * 1024);
#pragma unroll
        for (int t = 0; t < TILES; ++t) S[t][p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q[t][c], S[t][p], 0, 0, 0);
      }
    }
    // V is requested before the softmax, whose instructions hide it; the empty asm
    // keeps the compiler from moving the reads down to their use
    uint4 V[kRowsPages][NK];
#pragma unroll
    for (int p = 0; p < kRowsPages; ++p)
#pragma unroll
      for (int i = 0; i < NK; ++i) V[p][i] = *(const uint4*)(base + (p * 2 * NK + NK + i) * 1024);
    asm volatile("" ::: "memory");
    const bool whole = i1 <= span.all_last && (i1 < full_sinks || i0 >= span.all_first);
    if (EDGE || !whole) {
#pragma unroll
      for (int p = 0; p < kRowsPages; ++p) {
        const int t0 = b.page(min(i0 + p, b.n_pages - 1)) * kPage + 4 * grp;
        const bool ok = !EDGE || ((there >> p) & 1);
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const bool seen = ok & row[t].sees(b, t0 + v);
            S[t][p][v] = seen ? S[t][p][v] : -INFINITY;  // a select, no branch
          }
      }
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      float mx = -INFINITY;
#pragma unroll
      for (int p = 0; p < kRowsPages; ++p)
#pragma unroll
        for (int v = 0; v < 4; ++v) mx = fmaxf(mx, S[t][p][v]);
      mx = max4(mx * a.scale_log2);
      float m = m_run[t];
      if (__any(mx - m > rise)) {
        m = mx - m <= kRise + kRowsDown ? m : fabsf(mx) > kFar ? mx : mx - kRowsDown;
        const float alpha = __builtin_amdgcn_exp2f(m_run[t] - m);
        m_run[t] = m;
        l_run[t] *= alpha;
#pragma unroll
        for (int n = 0; n < 2 * NK; ++n) O[t][n] *= alpha;
        if (__any(fabsf(m) > kFar && m != kLowest)) {
          // here in every step from now on: exponents first, in the scores' units and from 0
#pragma unroll
          for (int p = 0; p < kRowsPages; ++p) {
            round_exponents(S[t][p], a.scale_log2, m);
            S[t][p] *= 1.f / a.scale_log2;
          }
          m = 0.f;
          rise = -INFINITY;
        }
      }
#pragma unroll
      for (int p = 0; p < kRowsPages; ++p)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float e = __builtin_amdgcn_exp2f(S[t][p][v] * a.scale_log2 - m);
          l_run[t] += e;
          P[t][p >> 1][(p & 1) * 4 + v] = (_Float16)e;
        }
    }
    uint4 keep[kRowsPages];
    if constexpr (EDGE) {
#pragma unroll
      for (int p = 0; p < kRowsPages; ++p) {
        const uint2 k = keep16(b, b.page(min(i0 + p, b.n_pages - 1)) * kPage + 4 * grp, (there >> p) & 1);
        keep[p] = uint4{k.x, k.y, k.x, k.y};
      }
    }
    // two pages per MFMA: k = 8 grp + 4 b + u is token 4 grp + u of page 2 h + b
#pragma unroll
    for (int h = 0; h < kRowsPages / 2; ++h)
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        uint4 va = V[2 * h][i], vb = V[2 * h + 1][i];
        if constexpr (EDGE) {
          va = both(va, keep[2 * h]);
          vb = both(vb, keep[2 * h + 1]);
        }
        const f16x8 v0 = __builtin_bit_cast(f16x8, uint4{va.x, va.y, vb.x, vb.y});
        const f16x8 v1 = __builtin_bit_cast(f16x8, uint4{va.z, va.w, vb.z, vb.w});
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
          O[t][2 * i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, P[t][h], O[t][2 * i], 0, 0, 0);
          O[t][2 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, P[t][h], O[t][2 * i + 1], 0, 0, 0);
        }
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // step st has been read (see arrive)
  };
  auto clean = [&](int st) {
    const int i0 = (st0 + st) * kRowsPages, i1 = i0 + kRowsPages - 1;
    return there == (1u << kRowsPages) - 1 && i1 <= live_last && (i1 < full_sinks || i0 >= live_first);
  };
  // Clean steps and those at an edge in loops of their own: in one loop the
  // outputs' registers would be moved about between the two bodies.
  int st = 0;
  if (n_st > 0) arrive(0);
  while (st < n_st) {
    if (!on) {
      if (++st < n_st) arrive(st);
      continue;
    }
    while (st < n_st && !clean(st)) {
      step(st, std::true_type{});
      if (++st < n_st) arrive(st);
    }
    while (st < n_st && clean(st)) {
      step(st, std::false_type{});
      if (++st < n_st) arrive(st);
    }
  }

#pragma unroll
  for (int t = 0; t < TILES; ++t) {
    const int i = w0 + t * 16 + r16;
    const float l = sum4(l_run[t]);
    if (i >= b.n_v) continue;
    const int v = b.v0 + i;
    if (splits > 1) {
      const size_t slot = part_slot(a, b, v, head, blockIdx.z);
#pragma unroll
      for (int n = 0; n < NK; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *(float4*)(part_o + slot * HD + 32 * n + 8 * grp + 4 * e) =
              make_float4(O[t][2 * n][2 * e], O[t][2 * n + 1][2 * e], O[t][2 * n][2 * e + 1], O[t][2 * n + 1][2 * e + 1]);
      if (grp == 0) *(float2*)(part_ml + slot * 2) = make_float2(m_run[t], l);
      continue;
    }
    const float inv = l > 0.f ? 1.f / l : l;
#pragma unroll
    for (int n = 0; n < NK; ++n) {
      f16x8 x;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        x[2 * u] = (_Float16)(O[t][2 * n][u] * inv);
        x[2 * u + 1] = (_Float16)(O[t][2 * n + 1][u] * inv);
      }
      *(f16x8*)out_at<_Float16, HD>(a, b.r0 + v / a.group, head * a.group + v % a.group, 32 * n + 8 * grp) = x;
    }
  }
}

// Row i of sequence (item) s, -1 for none.
__device__ __forceinline__ int join_row(const WindowArgs& a, int s, int i) {
  const int r0 = min(max(a.row_offsets[s], 0), a.rows), r1 = min(max(a.row_offsets[s + 1], r0), a.rows);
  return i < r1 - r0 ? r0 + i : -1;
}
__device__ __forceinline__ int join_row(const WindowStepArgs& a, int s, int i) {
  return i < a.item[s].rows ? a.item[s].row0 + i : -1;
}

// Joins the splits' states, a workgroup for each (row, query head), a quarter of
// the splits for each of its waves.  grid (rows of a sequence, sequence, query head).
template <typename T, int HD, typename A>
__global__ __launch_bounds__(256) void k_window_join(A a, int splits, const float* part_o, const float* part_ml) {
  constexpr int N = HD / 64;
  __shared__ float s_o[4][HD];
  const int s = blockIdx.y, qh = blockIdx.z, heads = a.n_heads * a.group;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int row = join_row(a, s, blockIdx.x);
  if (row < 0) return;
  const size_t slot = (size_t)row * heads + qh, stride = (size_t)a.rows * heads;
  float2 ml = make_float2(kLowest, 0.f);
  if (lane < splits) ml = *(const float2*)(part_ml + (slot + lane * stride) * 2);
  float p[kMaxSplits / 4][N];
#pragma unroll
  for (int i = 0; i < kMaxSplits / 4; ++i) {
    const int g = min(wave + 4 * i, splits - 1);
    if (4 * i >= splits) break;
#pragma unroll
    for (int n = 0; n < N; ++n) p[i][n] = part_o[(slot + g * stride) * HD + lane * N + n];
  }
  float top = ml.x, L;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  // a split that saw nothing has weight 0: it may have written no output
  const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
  L = f * ml.y;
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) L += __shfl_xor(L, off);
  float o[N] = {};
#pragma unroll
  for (int i = 0; i < kMaxSplits / 4; ++i) {
    const int g = wave + 4 * i;
    if (g >= splits) break;
    const float w = __shfl(f, g);
#pragma unroll
    for (int n = 0; n < N; ++n) o[n] += w == 0.f ? 0.f : w * p[i][n];
  }
#pragma unroll
  for (int n = 0; n < N; ++n) s_o[wave][lane * N + n] = o[n];
  __syncthreads();
  if (threadIdx.x < HD) {
    const int d = threadIdx.x;
    const float x = (s_o[0][d] + s_o[1][d]) + (s_o[2][d] + s_o[3][d]);
    *out_at<T, HD>(a, row, qh, d) = (T)(x * (L > 0.f ? 1.f / L : L));
  }
}

// The same by a wave for each (row, query head), for at most sixteen splits: after the
// kernel of many rows, whose pairs fill the chip by themselves (300 rows of 32 heads
// over 700 tokens in five splits 29.1 us with workgroups, 25.7 with waves; one row over
// 1028 tokens of 32 heads, after the kernel of few, 9.3 and 10.0).
// grid (rows of a sequence, sequence, query heads / 4).
constexpr int kWaveSplits = 16;
template <int HD, typename A>
__global__ __launch_bounds__(256) void k_window_join_wave(A a, int splits, const float* part_o, const float* part_ml) {
  constexpr int N = HD / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int heads = a.n_heads * a.group, qh = blockIdx.z * 4 + wave;
  const int row = join_row(a, blockIdx.y, blockIdx.x);
  if (row < 0 || qh >= heads) return;
  const size_t slot = (size_t)row * heads + qh, stride = (size_t)a.rows * heads;
  float2 ml = make_float2(kLowest, 0.f);
  if (lane < splits) ml = *(const float2*)(part_ml + (slot + lane * stride) * 2);
  float p[kWaveSplits][N];
#pragma unroll
  for (int i = 0; i < kWaveSplits; ++i) {
#pragma unroll
    for (int n = 0; n < N; ++n) p[i][n] = i < splits ? part_o[(slot + i * stride) * HD + lane * N + n] : 0.f;
  }
  float top = ml.x, L;
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  // a split that saw nothing has weight 0: it may have written no output
  const float f = ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
  L = f * ml.y;
#pragma unroll
  for (int off = 8; off >= 1; off >>= 1) L += __shfl_xor(L, off);
  L = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(L)));
  const float inv = L > 0.f ? 1.f / L : L;
  float o[N] = {};
#pragma unroll
  for (int i = 0; i < kWaveSplits; ++i) {
    const float g = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i));
#pragma unroll
    for (int n = 0; n < N; ++n) o[n] += i < splits && g != 0.f ? g * p[i][n] : 0.f;
  }
#pragma unroll
  for (int n = 0; n < N; ++n) *out_at<_Float16, HD>(a, row, qh, lane * N + n) = (_Float16)(o[n] * inv);
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
