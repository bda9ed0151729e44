// Copies of cache pages, and the reordering of beams' pages (gfx950).
//
// Bound by HBM.  A workgroup of a copy moves 16 KiB of one source page of one layer, four
// 16-byte loads in flight per thread, and stores what it read to every page that
// stands next to it in the list with the same source, so a page that goes to
// several places is read once: 65 pages of 4 layers to 7 places each (545 MB) take
// 114 us, 4.8 TB/s (read for every place 202 us), 700 pages of 2 layers moved one by
// one (918 MB) 194 us, 4.7 TB/s; a large copy reaches 4.9.
#include "tss_internal.h"
#include <type_traits>

namespace tss {

constexpr int kCopyThreads = 256, kCopyLoads = 4;
constexpr int kCopySlice = kCopyThreads * kCopyLoads * 16;
constexpr int kReorderPiece = kCopyThreads * 16;
typedef unsigned Piece __attribute__((ext_vector_type(4)));

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


// f(integral_constant<int, p>) for p = 0 .. B - 1: the beams' bytes stay in registers only
// where their index is a constant, and the compiler does not unroll a loop around one of heirs.
template <int B, int P = 0, typename F>
__device__ __forceinline__ void each_beam(F f) {
  if constexpr (P < B) {
    f(std::integral_constant<int, P>{});
    each_beam<B, P + 1>(f);
  }
}

// Reordering: sequence b of a group becomes sequence parents[b], in place.  A thread
// reads its 16 bytes of every page that is taken over before it writes the first of
// those that change, so an exchange needs no other memory and no barrier, and a page
// that several beams take over is read once.  Bound by HBM: 8 groups of 8 beams, three of
// which go on, of 250 to 500 tokens in 4 layers (379 MB) take 77 us, 4.9 TB/s; with two or
// four pieces a thread it is the same, and with the beams' bytes in scratch memory, where the
// struct type uint4 or a loop over them puts them, it was 118.
// grid (pieces of a page x pages, group, layer)
template <int B>
__global__ __launch_bounds__(kCopyThreads, B <= 8 ? 8 : B <= 16 ? 6 : 3) void k_reorder_pages(ReorderArgs a,
                                                                                          int pieces) {
  const int g = blockIdx.y, l = blockIdx.z, lane = threadIdx.x & 63;
  if (!((a.layers[l >> 6] >> (l & 63)) & 1ull)) return;
  const int first = a.shared ? min(max(a.shared[g], 0), a.table_stride) : a.first;
  const int pg = first + (int)(blockIdx.x / pieces);
  if (pg >= a.table_stride) return;
  // lane b: beam b of the group
  const int beam = min(lane, a.n_beams - 1), at_seq = g * a.n_beams + beam;
  const int seq = a.parents ? at_seq : a.seq[beam];
  int parent = a.parents ? a.parents[at_seq] : a.parent[beam];
  const int id = a.page_table[(size_t)seq * a.table_stride + pg];
  const int len = a.parents ? a.lengths[at_seq] : a.length[beam];
  const bool there = (unsigned)id < (unsigned)a.n_pages;
  const uint64_t full = __ballot(lane < a.n_beams && there && pg * kPage < len);  // a page to take
  const bool moves = lane < a.n_beams && there && (unsigned)parent < (unsigned)a.n_beams && parent != lane &&
                     ((full >> (parent & 63)) & 1);
  if (!moves) parent = -1;
  uint8_t* at = a.pages + (size_t)l * a.layer_bytes + (size_t)(blockIdx.x % pieces) * kReorderPiece + threadIdx.x * 16;
  uint64_t heirs[B];
  Piece v[B];
  each_beam<B>([&](auto i) {
    constexpr int p = decltype(i)::value;
    heirs[p] = __ballot(parent == p);
    if (heirs[p]) v[p] = *(const Piece*)(at + (size_t)__builtin_amdgcn_readlane(id, p) * a.page_bytes);
  });
  each_beam<B>([&](auto i) {
    constexpr int p = decltype(i)::value;
    for (uint64_t m = heirs[p]; m; m &= m - 1) {
      const int to = __builtin_amdgcn_readlane(id, __builtin_ctzll(m));
      if (to != __builtin_amdgcn_readlane(id, p)) *(Piece*)(at + (size_t)to * a.page_bytes) = v[p];
    }
  });
}

static int64_t pieces_of(const ReorderArgs& a) { return a.page_bytes / kReorderPiece; }
static int64_t pages_of(const ReorderArgs& a) { return ((int64_t)a.max_own + kPage - 1) / kPage; }

bool reorder_fits(const ReorderArgs& a) {
  return a.n_groups <= 65535 && pieces_of(a) * pages_of(a) <= INT32_MAX / kCopyThreads;
}

hipError_t launch_reorder(const ReorderArgs& a, hipStream_t s) {
  const int64_t pieces = pieces_of(a);
  // a page has whole pieces: a head's K alone is 2 KiB, and V as much
  if (a.page_bytes % kReorderPiece != 0 || a.table_stride > INT32_MAX / kPage || a.n_groups < 1 || a.n_beams < 1 ||
      a.n_beams > kMaxBeams || (!a.parents && a.n_groups != 1) || a.first < 0 || a.n_layers < 1 || a.n_layers > kMaxLayers || a.max_own < 1 || !reorder_fits(a))
    return hipErrorInvalidValue;
  const dim3 grid(pieces * pages_of(a), a.n_groups, a.n_layers), block(kCopyThreads);
  if (a.n_beams <= 4)
    TSS_LAUNCH(k_reorder_pages<4>, grid, block, 0, s, a, (int)pieces);
  else if (a.n_beams <= 8)
    TSS_LAUNCH(k_reorder_pages<8>, grid, block, 0, s, a, (int)pieces);
  else if (a.n_beams <= 16)
    TSS_LAUNCH(k_reorder_pages<16>, grid, block, 0, s, a, (int)pieces);
  else
    TSS_LAUNCH(k_reorder_pages<32>, grid, block, 0, s, a, (int)pieces);
  return hipGetLastError();
}

}  // namespace tss
