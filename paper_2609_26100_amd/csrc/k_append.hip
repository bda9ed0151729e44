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
#include "../../include/tss.h"
#include "tss_internal.h"

#include <algorithm>

namespace tss {

namespace {

constexpr int kAppendThreads = 256;

template <int TYPE> struct In;  // eight elements
template <> struct In<TSS_T_F32> {
  using T = float;
  static constexpr int size = 4;
  __device__ static void load(const void* p, float* x) {
    const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
};
template <> struct In<TSS_T_F16> {
  static constexpr int size = 2;
  __device__ static void load(const void* p, float* x) {
    typedef _Float16 h8 __attribute__((ext_vector_type(8)));
    const h8 h = *(const h8*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
  }
};
template <> struct In<TSS_T_BF16> {
  static constexpr int size = 2;
  __device__ static void load(const void* p, float* x) {
    const uint4 v = *(const uint4*)p;
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
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
  constexpr int ES = In<TYPE>::size, HALF = HD / 2, C = HALF / 8, VC = HD / 8;
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
  int id = -1;
  if (page < a.table_stride) id = a.page_table[(size_t)s * a.table_stride + page];
  const bool there = (unsigned)id < (unsigned)a.n_pages;
  T* const kpage = (T*)a.kv_pages + (size_t)(there ? id : 0) * 2 * a.n_heads * (kPage * HD);
  T* const vpage = kpage + (size_t)a.n_heads * (kPage * HD);

  for (int i = tid; i < nt * HALF; i += kAppendThreads) {
    const int t = i / HALF, j = i % HALF;
    float2 cs = make_float2(1.f, 0.f);
    if (a.rotate) {
      const int pos = a.positions ? a.positions[row0 + t] : (int)(lo64 + t);
      const double x = (double)pos * a.turns[j];
      const float y = 2.f * (float)(x - rint(x));
      cs = make_float2(cospif(y), sinpif(y));
    }
    s_cs[t][j] = cs;
  }
  __syncthreads();

  const int all = a.n_q_heads + 2 * a.n_heads;
  const int u0 = blockIdx.z * units, u1 = min(u0 + units, all);
  // q and K: item (head, token, chunk of 8 pairs)
  const int rot0 = min(u0, a.n_q_heads + a.n_heads), rot1 = min(u1, a.n_q_heads + a.n_heads);
  for (int i = tid; i < (rot1 - rot0) * nt * C; i += kAppendThreads) {
    const int c = i % C, t = i / C % nt, u = rot0 + i / (C * nt);
    const bool is_q = u < a.n_q_heads;
    const int h = is_q ? u : u - a.n_q_heads, row = row0 + t;
    if (!is_q && !there) continue;
    const uint8_t* from = (const uint8_t*)(is_q ? a.q : a.k) +
                          ((size_t)row * (is_q ? a.q_stride : a.k_stride) + (size_t)h * HD + c * 8) * ES;
    float x[8], y[8], z[8];
    In<TYPE>::load(from, x);
    In<TYPE>::load(from + HALF * ES, y);
    if (a.rotate) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 cs = s_cs[t][c * 8 + e];
        z[e] = x[e] * cs.x - y[e] * cs.y;
        y[e] = y[e] * cs.x + x[e] * cs.y;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = x[e];
    }
    T* to = (is_q ? (T*)a.q_out + (size_t)row * a.q_out_stride + (size_t)h * HD
                  : kpage + (size_t)h * (kPage * HD) + (t0 + t) * HD) + c * 8;
    store8(to, z);
    store8(to + HALF, y);
  }
  // V: item (head, group of four tokens, chunk of 8 dimensions)
  if (!there) return;
  const int v0 = max(u0, a.n_q_heads + a.n_heads), v1 = u1;
  const int g0 = t0 / 4, groups = (t0 + nt - 1) / 4 - g0 + 1;
  for (int i = tid; i < (v1 - v0) * groups * VC; i += kAppendThreads) {
    const int c = i % VC, g = g0 + i / VC % groups, h = v0 + i / (VC * groups) - a.n_q_heads - a.n_heads;
    float x[4][8];
    const int first = max(g * 4, t0), last = min(g * 4 + 4, t0 + nt);  // its new tokens
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = min(max(g * 4 + e, first), last - 1);
      In<TYPE>::load((const uint8_t*)a.v + ((size_t)(row0 + t - t0) * a.v_stride + (size_t)h * HD + c * 8) * ES, x[e]);
    }
    T* to = vpage + (size_t)h * (kPage * HD) + (g * HD + c * 8) * 4;
    if (last - first == 4) {
#pragma unroll
      for (int d = 0; d < 8; d += 2) {
        const float w[8] = {x[0][d],     x[1][d],     x[2][d],     x[3][d],
                            x[0][d + 1], x[1][d + 1], x[2][d + 1], x[3][d + 1]};
        store8(to + d * 4, w);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (g * 4 + e >= first && g * 4 + e < last)
#pragma unroll
          for (int d = 0; d < 8; ++d) to[d * 4 + e] = (T)x[e][d];
    }
  }
}

template <typename T, int HD, int TYPE>
hipError_t launch_typed(const AppendArgs& a, hipStream_t s) {
  const int all = a.n_q_heads + 2 * a.n_heads, tokens = std::min(a.max_rows, kPage);
  const int units = std::max(1, kAppendThreads * 4 / (HD / 16 * tokens));
  const dim3 grid((a.max_rows + 14) / kPage + 1, a.n_seqs, (all + units - 1) / units);
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
