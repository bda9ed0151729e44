// Copies of cache pages (gfx950).
#include "tss_internal.h"

namespace tss {

// One workgroup per (copy, layer), 16 bytes a thread.
__global__ __launch_bounds__(256) void k_copy_pages(CopyArgs a) {
  uint8_t* layer = a.pages + (size_t)blockIdx.y * a.layer_bytes;
  const uint4* src = (const uint4*)(layer + (size_t)a.src[blockIdx.x] * a.page_bytes);
  uint4* dst = (uint4*)(layer + (size_t)a.dst[blockIdx.x] * a.page_bytes);
  for (size_t i = threadIdx.x; i < a.page_bytes / 16; i += 256) dst[i] = src[i];
}

hipError_t launch_copy_pages(const CopyArgs& a, hipStream_t s) {
  if (a.n < 1 || a.n > kCopyPairs || a.n_layers < 1 || a.n_layers > 65535) return hipErrorInvalidValue;
  TSS_LAUNCH(k_copy_pages, dim3(a.n, a.n_layers), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace tss
