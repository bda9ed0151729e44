// Attention with a sliding window and sinks over the paged KV cache (gfx950).
#include "../../include/tss.h"
#include "tss_internal.h"

namespace tss {

// One wave per (row, query head); a lane holds HD / 64 dimensions.
template <typename T, int HD>
__global__ __launch_bounds__(256) void k_window(WindowArgs a) {
  constexpr int N = HD / 64;
  const int lane = threadIdx.x & 63;
  const int qh = blockIdx.y * 4 + (threadIdx.x >> 6), kvh = qh / a.group;
  if (qh >= a.n_heads * a.group) return;
  const int s = blockIdx.x / a.max_rows, i = blockIdx.x % a.max_rows;
  const int r0 = max(a.row_offsets[s], 0), r1 = min(a.row_offsets[s + 1], a.rows);
  const int r = r0 + i;
  if (r >= r1) return;
  const int len = min(min(a.lengths[s], a.max_length), a.table_stride * kPage);
  const int p = len - (r1 - r0) + i;
  float q[N], o[N], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    q[n] = (float)((const T*)a.q)[(size_t)r * a.q_stride + (size_t)qh * HD + lane * N + n] * a.scale_log2;
    o[n] = 0.f;
  }
  for (int t = 0; t <= p; ++t) {
    if (a.window > 0 && t >= a.sinks && t <= p - a.window) {
      t = p - a.window;
      continue;
    }
    const int page = a.page_table[(size_t)s * a.table_stride + t / kPage], c = t % kPage;
    if (page < 0 || page >= a.n_pages) continue;
    const T* k = (const T*)a.kv_pages + (((size_t)page * 2) * a.n_heads + kvh) * (kPage * HD);
    const T* v = k + (size_t)a.n_heads * (kPage * HD);
    float d = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) d += q[n] * (float)k[c * HD + lane * N + n];
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) d += __shfl_xor(d, off);
    const float mx = fmaxf(m, d), f = exp2f(m - mx), e = exp2f(d - mx);
    m = mx;
    l = l * f + e;
#pragma unroll
    for (int n = 0; n < N; ++n) o[n] = o[n] * f + e * (float)v[(c / 4) * HD * 4 + (lane * N + n) * 4 + c % 4];
  }
#pragma unroll
  for (int n = 0; n < N; ++n)
    ((T*)a.o)[(size_t)r * a.o_stride + (size_t)qh * HD + lane * N + n] = (T)(l > 0.f ? o[n] / l : 0.f);
}

hipError_t launch_window(bool f16, int head_dim, const WindowArgs& a, hipStream_t s) {
  const dim3 grid(a.n_seqs * a.max_rows, (a.n_heads * a.group + 3) / 4);
  if (f16 && head_dim == 128)
    TSS_LAUNCH((k_window<_Float16, 128>), grid, dim3(256), 0, s, a);
  else if (f16)
    TSS_LAUNCH((k_window<_Float16, 64>), grid, dim3(256), 0, s, a);
  else if (head_dim == 128)
    TSS_LAUNCH((k_window<float, 128>), grid, dim3(256), 0, s, a);
  else
    TSS_LAUNCH((k_window<float, 64>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace tss
