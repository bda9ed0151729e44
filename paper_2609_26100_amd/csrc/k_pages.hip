// Copies of cache pages, and the reordering of beams' pages (gfx950).
//
// Bound by HBM.  A workgroup of a copy moves 16 KiB of one source page of one layer, four
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


// Reordering: sequence b of a group becomes sequence parents[b], in place.  A thread
// reads its 16 bytes of every page that is taken over before it writes the first of
// those that change, so an exchange needs no other memory and no barrier, and a page
// that several beams take over is read once.  grid (slices of a page x pages, group, layer)
template <int B>
__global__ __launch_bounds__(kCopyThreads) void k_reorder_pages(ReorderArgs a, int slices) {
  const int g = blockIdx.y, l = blockIdx.z, lane = threadIdx.x & 63;
  if (!((a.layers[l >> 6] >> (l & 63)) & 1ull)) return;
  const int first = a.shared ? min(max(a.shared[g], 0), a.table_stride) : 0;
  const int pg = first + (int)(blockIdx.x / slices);
  if (pg >= a.table_stride) return;
  // lane b: beam b of the group
  const int seq = g * a.n_beams + min(lane, a.n_beams - 1);
  int parent = a.parents[seq];
  const int id = a.page_table[(size_t)seq * a.table_stride + pg];
  const int len = a.lengths[seq];
  const bool there = (unsigned)id < (unsigned)a.n_pages;
  const uint64_t full = __ballot(lane < a.n_beams && there && pg * kPage < len);  // a page to take
  const bool moves = lane < a.n_beams && there && (unsigned)parent < (unsigned)a.n_beams && parent != lane &&
                     ((full >> (parent & 63)) & 1);
  if (!moves) parent = -1;
  const size_t at = (size_t)(blockIdx.x % slices) * (kCopyThreads * 16) + threadIdx.x * 16;
  uint8_t* layer = a.pages + (size_t)l * a.layer_bytes + at;
  uint64_t heirs[B];
  uint4 v[B];
#pragma unroll
  for (int p = 0; p < B; ++p) {
    heirs[p] = __ballot(parent == p);
    if (heirs[p]) v[p] = *(const uint4*)(layer + (size_t)__builtin_amdgcn_readlane(id, p) * a.page_bytes);
  }
#pragma unroll
  for (int p = 0; p < B; ++p)
    for (uint64_t m = heirs[p]; m; m &= m - 1) {
      const int b = __builtin_ctzll(m), to = __builtin_amdgcn_readlane(id, b);
      if (to != __builtin_amdgcn_readlane(id, p)) *(uint4*)(layer + (size_t)to * a.page_bytes) = v[p];
    }
}

static int64_t slices_of(const ReorderArgs& a) { return a.page_bytes / (kCopyThreads * 16); }
static int64_t pages_of(const ReorderArgs& a) { return ((int64_t)a.max_own + kPage - 1) / kPage; }

bool reorder_fits(const ReorderArgs& a) {
  return a.n_groups <= 65535 && slices_of(a) * pages_of(a) <= INT32_MAX / kCopyThreads;
}

hipError_t launch_reorder(const ReorderArgs& a, hipStream_t s) {
  const int64_t slices = slices_of(a), pages = pages_of(a);
  // a page has whole slices: a head's K alone is 2 KiB, and V as much
  if (a.page_bytes % (kCopyThreads * 16) != 0 || a.table_stride > INT32_MAX / kPage || a.n_groups < 1 ||
      a.n_beams < 1 || a.n_beams > 32 || a.n_layers < 1 || a.n_layers > kMaxLayers || pages < 1 || !reorder_fits(a))
    return hipErrorInvalidValue;
  const dim3 grid(slices * pages, a.n_groups, a.n_layers), block(kCopyThreads);
  if (a.n_beams <= 4)
    TSS_LAUNCH(k_reorder_pages<4>, grid, block, 0, s, a, (int)slices);
  else if (a.n_beams <= 8)
    TSS_LAUNCH(k_reorder_pages<8>, grid, block, 0, s, a, (int)slices);
  else if (a.n_beams <= 16)
    TSS_LAUNCH(k_reorder_pages<16>, grid, block, 0, s, a, (int)slices);
  else
    TSS_LAUNCH(k_reorder_pages<32>, grid, block, 0, s, a, (int)slices);
  return hipGetLastError();
}

}  // namespace tss
