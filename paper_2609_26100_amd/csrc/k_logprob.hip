// Log probabilities of given tokens, entropy and alternatives (gfx950).
//
// With m = max x, S = sum e^(x - m) and T = sum (x - m) e^(x - m) of a row:
//   logprob = x - m - ln S,  entropy = ln S - T / S.
#include "../../include/tss.h"
#include "tss_internal.h"


namespace tss {

template <int TYPE>
__device__ __forceinline__ float load_logit(const void* p, int i) {
  if constexpr (TYPE == TSS_T_F32) return ((const float*)p)[i];
  if constexpr (TYPE == TSS_T_F16) return (float)((const _Float16*)p)[i];
  return __uint_as_float((unsigned)((const uint16_t*)p)[i] << 16);
}

// Unsigned key in the order of the logits: larger values have larger keys,
// -0 and +0 the same one, NaN the largest.
__device__ __forceinline__ unsigned order_key(float x) {
  if (x != x) return 0xfffffffeu;
  const unsigned b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Key of (logit, token): the lower token first among equal logits.
__device__ __forceinline__ unsigned long long pair_key(float x, int i) {
  return ((unsigned long long)order_key(x) << 32) | (unsigned)~i;
}

template <typename F, typename V>
__device__ __forceinline__ V block_reduce(V v, V* lds, F f) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = f(v, __shfl_xor(v, off));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
  for (int w = 1; w < 4; ++w) v = f(v, lds[w]);
  return v;
}

// One workgroup per row.
template <int TYPE>
__global__ __launch_bounds__(256) void k_logprobs(LogprobArgs a) {
  __shared__ float red[4];
  __shared__ int redi[4];
  __shared__ unsigned long long redk[4];
  const int r = blockIdx.x, V = a.vocab;
  constexpr int ES = TYPE == TSS_T_F32 ? 4 : 2;
  const void* x = (const uint8_t*)a.x + (size_t)r * a.stride * ES;
  float m = -INFINITY;
  for (int i = threadIdx.x; i < V; i += 256) m = fmaxf(m, load_logit<TYPE>(x, i));
  m = block_reduce(m, red, [](float p, float q) { return fmaxf(p, q); });
  const float base = m == -INFINITY ? 0.f : m;
  float S = 0.f, T = 0.f;
  for (int i = threadIdx.x; i < V; i += 256) {
    const float d = load_logit<TYPE>(x, i) - base, e = expf(d);
    S += e;
    T += e == 0.f ? 0.f : d * e;
  }
  S = block_reduce(S, red, [](float p, float q) { return p + q; });
  T = block_reduce(T, red, [](float p, float q) { return p + q; });
  const float ln = logf(S);
  // x - m - ln S; a row without a token left has none to share
  auto lp = [&](float v) { return S == 0.f ? -INFINITY : v - base - ln; };
  if (threadIdx.x == 0 && a.entropy) a.entropy[r] = S == 0.f ? 0.f : ln - T / S;
  for (int t = 0; t < a.n_tokens; ++t) {
    const int tok = a.tokens[(size_t)r * a.n_tokens + t];
    const bool in = tok >= 0 && tok < V;
    const float xt = in ? load_logit<TYPE>(x, tok) : 0.f;
    const unsigned long long k = pair_key(xt, tok);
    int n = 0;
    for (int i = threadIdx.x; i < V; i += 256) n += pair_key(load_logit<TYPE>(x, i), i) > k;
    n = block_reduce(n, redi, [](int p, int q) { return p + q; });
    if (threadIdx.x == 0) {
      if (a.logprob) a.logprob[(size_t)r * a.n_tokens + t] = in ? lp(xt) : NAN;
      if (a.rank) a.rank[(size_t)r * a.n_tokens + t] = in ? n : -1;
    }
  }
  unsigned long long last = ~0ull;
  for (int t = 0; t < a.top_k; ++t) {
    unsigned long long k = 0;
    for (int i = threadIdx.x; i < V; i += 256) {
      const unsigned long long c = pair_key(load_logit<TYPE>(x, i), i);
      if (c < last && c > k) k = c;
    }
    last = block_reduce(k, redk, [](unsigned long long p, unsigned long long q) { return p > q ? p : q; });
    const int i = (int)~(unsigned)last;
    if (threadIdx.x == 0) {
      if (a.top_logprob) a.top_logprob[(size_t)r * a.top_k + t] = lp(load_logit<TYPE>(x, i));
      if (a.top_token) a.top_token[(size_t)r * a.top_k + t] = i;
    }
  }
}

hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t s) {
  if (a.rows < 1 || a.vocab < 1) return hipErrorInvalidValue;
  if (a.type == TSS_T_F32)
    TSS_LAUNCH(k_logprobs<TSS_T_F32>, dim3(a.rows), dim3(256), 0, s, a);
  else if (a.type == TSS_T_F16)
    TSS_LAUNCH(k_logprobs<TSS_T_F16>, dim3(a.rows), dim3(256), 0, s, a);
  else
    TSS_LAUNCH(k_logprobs<TSS_T_BF16>, dim3(a.rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace tss
