// Rows of logits and sums over a wave (gfx950), for the kernels that read logits.
#pragma once

#include "../../include/tss.h"
#include "tss_internal.h"

#include <type_traits>

namespace tss {

namespace {

template <int TYPE> struct Logit;
template <> struct Logit<TSS_T_F32> {
  static constexpr int size = 4;
  __device__ static float at(const void* p, size_t i) { return ((const float*)p)[i]; }
  __device__ static void spread(uint4 v, float* x) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
  }
};
template <> struct Logit<TSS_T_F16> {
  static constexpr int size = 2;
  __device__ static float at(const void* p, size_t i) { return (float)((const _Float16*)p)[i]; }
  __device__ static void spread(uint4 v, float* x) {
    typedef _Float16 h8 __attribute__((ext_vector_type(8)));
    const h8 h = __builtin_bit_cast(h8, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)h[e];
  }
};
template <> struct Logit<TSS_T_BF16> {
  static constexpr int size = 2;
  __device__ static float at(const void* p, size_t i) {
    return __uint_as_float((unsigned)((const uint16_t*)p)[i] << 16);
  }
  __device__ static void spread(uint4 v, float* x) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
};

// All lanes' values joined by f, for every lane (a scalar), in a fixed order, by
// DPP moves: no trip through LDS.  none: f's neutral value.
template <typename V, typename F>
__device__ __forceinline__ V wave_reduce(V v, V none, F f) {
  auto move = [&](auto ctrl, auto rows) {
    const int m = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v),
                                              decltype(ctrl)::value, decltype(rows)::value, 0xf, false);
    v = f(v, __builtin_bit_cast(V, m));
  };
  using std::integral_constant;
  move(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});  // from 1, 2, 4, 8 lanes before in the row
  move(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  move(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  move(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  move(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});  // a row's last lane to the next row
  move(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});  // lane 31 to the upper half
  return __builtin_bit_cast(V, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_reduce(v, 0.f, [](float p, float q) { return p + q; });
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_reduce(v, -INFINITY, [](float p, float q) { return fmaxf(p, q); });
}
__device__ __forceinline__ int wave_sum(int v) {
  return wave_reduce(v, 0, [](int p, int q) { return p + q; });
}
}  // namespace

}  // namespace tss
