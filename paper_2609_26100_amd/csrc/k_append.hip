// Rows appended to the paged KV cache, rotated to their positions (gfx950).
//
//   angle_j = position f_j;  (x_j, x_{j + hd/2}) -> (x_j c - x_{j + hd/2} s, x_{j + hd/2} c + x_j s)
//
// A workgroup takes the new rows of one page of a sequence (up to 16 slots) and some
// of the heads.  The cosines and sines of its rows go to LDS first, a thread each:
// position x f_j in turns in 64 bits, of which the whole turns are dropped, so that a
// position of 10^6 (where 32 bits leave an angle off by 0.06) loses nothing.  Then a
// thread has eight dimensions of each half of a head's row, of q or K, or, of V, eight
// dimensions of a group of four tokens, which the cache holds side by side: 16-byte
// loads and stores, except where only some of the four are new.
//
// Bound by HBM for many rows (3500 rows of 40 + 2 x 40 heads of 128, fp32 to fp16, 323 MB: 65.5 us,
// 4.9 TB/s), by a launch and three dependent loads for few (one row of 32 + 2 x 32 heads 5.7 us).
#include "../../include/tss.h"
#include "tss_internal.h"

#include <algorithm>

namespace tss {

namespace {

constexpr int kAppendThreads = 256;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Eight elements: as they are loaded, and in fp32.
template <int TYPE> struct Eight;
template <> struct Eight<TSS_T_F32> {
  static constexpr int size = 4;
  u32x4 w[2];
  __device__ void load(const void* p) {
    w[0] = ((const u32x4*)p)[0];
    w[1] = ((const u32x4*)p)[1];
  }
  __device__ float at(int e) const { return __uint_as_float(w[e / 4][e % 4]); }
};
template <> struct Eight<TSS_T_F16> {
  typedef _Float16 h8 __attribute__((ext_vector_type(8)));
  static constexpr int size = 2;
  h8 h;
  __device__ void load(const void* p) { h = *(const h8*)p; }
  __device__ float at(int e) const { return (float)h[e]; }
};
template <> struct Eight<TSS_T_BF16> {
  static constexpr int size = 2;
  u32x4 w;
  __device__ void load(const void* p) { w = *(const u32x4*)p; }
  __device__ float at(int e) const { return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16); }
};

// Eight elements to consecutive places, one rounding each.
__device__ __forceinline__ void store8(float* p, const float* x) {
  ((float4*)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  ((float4*)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(_Float16* p, const float* x) {
  typedef _Float16 h8 __attribute__((ext_vector_type(8)));
  h8 h;
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = (_Float16)x[e];
  *(h8*)p = h;
}

// grid (pages of a sequence's new rows, sequence, shares of the heads).  units: heads (of
// q, then K, then V) of a workgroup.
template <typename T, int HD, int TYPE>
__global__ __launch_bounds__(kAppendThreads) void k_append(AppendArgs a, int units) {
  using E = Eight<TYPE>;
  constexpr int ES = E::size, HALF = HD / 2, C = HALF / 8, VC = HD / 8;
  __shared__ float2 s_cs[kPage][HALF + 1];
  const int s = blockIdx.y, tid = threadIdx.x;
  const int r0 = min(max(a.row_offsets[s], 0), a.rows);
  const int r = min(max(a.row_offsets[s + 1], r0), a.rows) - r0;
  const int64_t p0 = (int64_t)a.lengths[s] - r;           // slot of row 0
  const int n = min(r, a.max_rows);
  // this block's slots [lo, hi)
  const int64_t page = max(p0, (int64_t)0) / kPage + blockIdx.x;
  const int64_t lo64 = max(max(p0, (int64_t)0), page * kPage), hi64 = min(p0 + n, page * kPage + kPage);
  if (lo64 >= hi64) return;
  const int t0 = (int)(lo64 - page * kPage), nt = (int)(hi64 - lo64);  // first token of the page, how many
  const int row0 = r0 + (int)(lo64 - p0);                              // row of token t0
  const int n_rot = a.n_q_heads + a.n_heads, u0 = blockIdx.z * units, u1 = min(u0 + units, n_rot + a.n_heads);
  const int rot0 = min(u0, n_rot), v0 = max(u0, n_rot);
  const int g0 = t0 / 4, groups = (t0 + nt - 1) / 4 - g0 + 1;
  const int rots = (min(u1, n_rot) - rot0) * nt * C, vs = (u1 - v0) * groups * VC;

  // item i of q and K: (head, token, chunk of 8 pairs); of V: (head, group of four tokens, chunk of
  // 8 dimensions).  A thread's first item is requested before anything that waits for positions and
  // page ids.
  struct Rot { E x, y; };
  struct Val { E x[4]; };
  auto load_rot = [&](int i, Rot& q) {
    if (i >= rots) return;
    const int c = i % C, t = i / C % nt, u = rot0 + i / (C * nt);
    const uint8_t* from =
        u < a.n_q_heads ? (const uint8_t*)a.q + ((size_t)(row0 + t) * a.q_stride + (size_t)u * HD + c * 8) * ES
                        : (const uint8_t*)a.k + ((size_t)(row0 + t) * a.k_stride + (size_t)(u - a.n_q_heads) * HD + c * 8) * ES;
    q.x.load(from);
    q.y.load(from + HALF * ES);
  };
  auto load_val = [&](int i, Val& q) {
    if (i >= vs) return;
    const int c = i % VC, g = g0 + i / VC % groups, h = v0 - n_rot + i / (VC * groups);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = min(max(g * 4 + e, t0), t0 + nt - 1);
      q.x[e].load((const uint8_t*)a.v + ((size_t)(row0 + t - t0) * a.v_stride + (size_t)h * HD + c * 8) * ES);
    }
  };
  Rot rot;
  Val val;
  load_rot(tid, rot);
  if (rots == 0) load_val(tid, val);

  int id = -1;
  if (page < a.table_stride) id = a.page_table[(size_t)s * a.table_stride + page];
  if (a.rotate && rots > 0) {
    for (int i = tid; i < nt * HALF; i += kAppendThreads) {
      const int t = i / HALF, j = i % HALF;
      const int pos = a.positions ? a.positions[row0 + t] : (int)(lo64 + t);
      const double x = (double)pos * a.turns[j];
      const float y = 2.f * (float)(x - rint(x));
      s_cs[t][j] = make_float2(cospif(y), sinpif(y));
    }
  }
  __syncthreads();
  const bool there = (unsigned)id < (unsigned)a.n_pages;
  T* const kpage = (T*)a.kv_pages + (size_t)(there ? id : 0) * 2 * a.n_heads * (kPage * HD);
  T* const vpage = kpage + (size_t)a.n_heads * (kPage * HD);

  for (int i = tid; i < rots; i += kAppendThreads) {
    if (i != tid) load_rot(i, rot);
    const Rot& q = rot;
    const int c = i % C, t = i / C % nt, u = rot0 + i / (C * nt);
    const bool is_q = u < a.n_q_heads;
    if (!is_q && !there) continue;
    float x[8], y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = q.x.at(e);
      y[e] = q.y.at(e);
    }
    if (a.rotate) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 cs = s_cs[t][c * 8 + e];
        const float z = x[e] * cs.x - y[e] * cs.y;
        y[e] = y[e] * cs.x + x[e] * cs.y;
        x[e] = z;
      }
    }
    T* to = (is_q ? (T*)a.q_out + (size_t)(row0 + t) * a.q_out_stride + (size_t)u * HD
                  : kpage + (size_t)(u - a.n_q_heads) * (kPage * HD) + (t0 + t) * HD) + c * 8;
    store8(to, x);
    store8(to + HALF, y);
  }
  if (!there) return;
  for (int i = tid; i < vs; i += kAppendThreads) {
    if (i != tid || rots > 0) load_val(i, val);
    const Val& q = val;
    const int c = i % VC, g = g0 + i / VC % groups, h = v0 - n_rot + i / (VC * groups);
    T* to = vpage + (size_t)h * (kPage * HD) + (g * HD + c * 8) * 4;
    if (g * 4 >= t0 && g * 4 + 4 <= t0 + nt) {
#pragma unroll
      for (int d = 0; d < 8; d += 2) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = q.x[e % 4].at(d + e / 4);
        store8(to + d * 4, w);
      }
    } else {  // some of the four are new
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (g * 4 + e >= t0 && g * 4 + e < t0 + nt)
#pragma unroll
          for (int d = 0; d < 8; ++d) to[d * 4 + e] = (T)q.x[e].at(d);
    }
  }
}

template <typename T, int HD, int TYPE>
hipError_t launch_typed(const AppendArgs& a, hipStream_t s) {
  const int all = a.n_q_heads + 2 * a.n_heads, tokens = std::min(a.max_rows, kPage);
  const int blocks = (a.max_rows + 14) / kPage + 1;
  // two items a thread: one row of 96 heads takes 5.6 us (one: 5.7, four: 7.3), 3500 rows of 120 65.4
  // (67, 72); 500 rows of 48 6.9 (6.2, 7.3)
  const int units = std::max(1, kAppendThreads * 2 / (HD / 16 * tokens));
  const dim3 grid(blocks, a.n_seqs, (all + units - 1) / units);
  TSS_LAUNCH((k_append<T, HD, TYPE>), grid, dim3(kAppendThreads), 0, s, a, units);
  return hipGetLastError();
}
template <typename T, int HD>
hipError_t launch_sized(const AppendArgs& a, hipStream_t s) {
  if (a.type == TSS_T_F32) return launch_typed<T, HD, TSS_T_F32>(a, s);
  if (a.type == TSS_T_F16) return launch_typed<T, HD, TSS_T_F16>(a, s);
  return launch_typed<T, HD, TSS_T_BF16>(a, s);
}

}  // namespace

bool append_fits(int n_q_heads, int n_heads, int n_seqs, int max_rows) {
  return n_seqs <= 65535 && (int64_t)n_q_heads + 2 * (int64_t)n_heads <= 65535 && max_rows <= (1 << 26);
}

hipError_t launch_append(bool f16, int head_dim, const AppendArgs& a, hipStream_t s) {
  if (a.max_rows < 1 || a.n_seqs < 1 || !append_fits(a.n_q_heads, a.n_heads, a.n_seqs, a.max_rows))
    return hipErrorInvalidValue;
  if (f16) return head_dim == 128 ? launch_sized<_Float16, 128>(a, s) : launch_sized<_Float16, 64>(a, s);
  return head_dim == 128 ? launch_sized<float, 128>(a, s) : launch_sized<float, 64>(a, s);
}

}  // namespace tss
