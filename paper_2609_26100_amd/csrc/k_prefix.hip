// Attention over the paged KV cache for sequences that share a prefix (gfx950).
//
// A wave for each (row, query head): one pass over the tokens with the running
// maximum and sum of the softmax, a lane for two dimensions.
#include "../../include/tss.h"
#include "tss_internal.h"

#include <algorithm>

namespace tss {

namespace {

template <typename T, int HD>
__global__ __launch_bounds__(64) void k_prefix(PrefixArgs a) {
  constexpr int N = HD / 64;
  const int s = blockIdx.y, qh = blockIdx.z, lane = threadIdx.x;
  const int r0 = min(max(a.row_offsets[s], 0), a.rows);
  const int r = min(max(a.row_offsets[s + 1], r0), a.rows) - r0;
  const int i = blockIdx.x;
  if (i >= min(r, a.max_rows)) return;
  const int len = max(0, min(min(a.lengths[s], a.max_length), a.table_stride * kPage));
  const int p = len - r + i, head = qh / a.group;
  // the group that holds the sequence
  int g = 0;
  while (a.group_offsets && g < a.n_groups && a.group_offsets[g + 1] <= s) ++g;
  int shared = 0, s0 = s;
  if (g < a.n_groups && (!a.group_offsets || a.group_offsets[g] <= s)) {
    s0 = a.group_offsets ? max(a.group_offsets[g], 0) : 0;
    shared = min(min(max(a.shared[g], 0), a.max_shared), a.table_stride);
  }
  const T* q = (const T*)a.q + (size_t)(r0 + i) * a.q_stride + (size_t)qh * HD;
  float x[N], o[N] = {}, m = -INFINITY, l = 0.f;
  for (int n = 0; n < N; ++n) x[n] = (float)q[n * 64 + lane];
  for (int t = 0; t <= p; ++t) {
    const int id = a.page_table[(size_t)(t / kPage < shared ? s0 : s) * a.table_stride + t / kPage];
    if ((unsigned)id >= (unsigned)a.n_pages) continue;
    const T* k = (const T*)a.kv_pages + ((size_t)id * 2 * a.n_heads + head) * (kPage * HD) + (t % kPage) * HD;
    const T* v = (const T*)a.kv_pages + ((size_t)(id * 2 + 1) * a.n_heads + head) * (kPage * HD) + (t % kPage) / 4 * HD * 4 + t % 4;
    float d = 0.f;
    for (int n = 0; n < N; ++n) d += x[n] * (float)k[n * 64 + lane];
    for (int w = 32; w > 0; w >>= 1) d += __shfl_xor(d, w);
    d *= a.scale_log2;
    const float top = fmaxf(m, d), f = m == -INFINITY ? 0.f : exp2f(m - top), e = exp2f(d - top);
    l = l * f + e;
    for (int n = 0; n < N; ++n) o[n] = o[n] * f + e * (float)v[(n * 64 + lane) * 4];
    m = top;
  }
  T* out = (T*)a.o + (size_t)(r0 + i) * a.o_stride + (size_t)qh * HD;
  for (int n = 0; n < N; ++n) out[n * 64 + lane] = (T)(l > 0.f ? o[n] / l : l);
}

template <typename T, int HD>
hipError_t launch_typed(const PrefixArgs& a, hipStream_t s) {
  TSS_LAUNCH((k_prefix<T, HD>), dim3(a.max_rows, a.n_seqs, a.n_heads * a.group), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace

bool prefix_fits(int n_heads, int group, int n_seqs, int max_rows, int n_groups, int max_group_rows) {
  return window_fits(n_heads, group, n_seqs, max_rows) && window_fits(n_heads, group, n_groups, max_group_rows);
}

size_t prefix_bytes(bool, int, int, int, int, int, int, int, int, int, int) { return 0; }

hipError_t launch_prefix(bool f16, int head_dim, const PrefixArgs& a, void*, hipStream_t s) {
  if (f16) return head_dim == 128 ? launch_typed<_Float16, 128>(a, s) : launch_typed<_Float16, 64>(a, s);
  return head_dim == 128 ? launch_typed<float, 128>(a, s) : launch_typed<float, 64>(a, s);
}

}  // namespace tss
