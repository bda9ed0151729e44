// Log probabilities of given tokens, entropy and alternatives (gfx950).
//
// With m = max x, S = sum e^(x - m) and T = sum (x - m) e^(x - m) of a row:
//   logprob = x - m - ln S,  entropy = ln S - T / S.
//
// A workgroup takes a chunk of a row, 32 logits a thread, into registers with
// 16-byte loads, so HBM is read once, and goes over the registers twice: for
// the maxima, and for S, T, the ranks and the candidates of the alternatives.
//   * Ranks: a token's rank is the number of logits that come before it, one
//     compare and a scalar popcount each; equal logits (the token's own, mostly)
//     are looked at again only by the waves that hold some.
//   * Alternatives: with W waves, every wave finds the ceil(k / W)-th largest of
//     its lanes' maxima (its top 16 bits, by bisection over ballots).  The least
//     of these has at least k logits at or above it, and few more: those
//     go to LDS, where each counts how many precede it.  Keys of (logit,
//     token) are unique, so the order in which they got there does not matter.
//     Where too many are equal for the LDS list, the k first are taken out one
//     by one instead.
// Rows of more than one chunk leave (m, S, T), counts and k keys for each chunk in the
// workspace and a second launch joins them.
#include "../../include/tss.h"
#include "tss_internal.h"

namespace tss {

namespace {

constexpr int kLpVals = 32;       // logits a thread holds
constexpr int kLpList = 512;      // candidates in LDS
constexpr int kLpTokens = TSS_LOGPROBS_MAX_TOKENS;
constexpr float kLog2e = 1.4426950408889634f;

typedef unsigned long long u64;

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

// Unsigned key in the order of the logits: larger values have larger keys,
// -0 and +0 the same one, NaN the largest; and back.
__device__ __forceinline__ unsigned order_key(float x) {
  if (x != x) return 0xfffffffeu;
  const unsigned b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(unsigned k) {
  if (k == 0xfffffffeu) return __uint_as_float(0x7fc00000u);
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
// Key of (logit, token): the lower token first among equal logits.  Never 0.
__device__ __forceinline__ u64 pair_key(float x, int i) { return ((u64)order_key(x) << 32) | (unsigned)~i; }

template <typename V, typename F>
__device__ __forceinline__ V wave_reduce(V v, F f) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = f(v, __shfl_xor(v, off));
  return v;
}

// What a row's (m, S, T) and a token's logit come to.
struct RowSums {
  float m, S, T;
  __device__ float base() const { return m == -INFINITY ? 0.f : m; }
  // a row without a token left has nothing to share out
  __device__ float logprob(float x) const { return S == 0.f ? -INFINITY : x - base() - logf(S); }
  __device__ float entropy() const { return S == 0.f ? 0.f : logf(S) - T / S; }
};

// A chunk's share of a row in the workspace (row-major over rows and chunks):
// floats m, S, T, then the token's counts, then k keys.
struct Parts {
  float* sums;    // [rows * chunks][3]
  int* counts;    // [rows * chunks][n_tokens]
  u64* keys;      // [rows * chunks][top_k], largest first, 0 where the chunk has fewer tokens
};

__device__ __forceinline__ void write_token(const LogprobArgs& a, size_t at, const RowSums& r, int tok, float xt,
                                            int rank) {
  const bool in = tok >= 0 && tok < a.vocab;
  if (a.logprob) a.logprob[at] = in ? r.logprob(xt) : __uint_as_float(0x7fc00000u);
  if (a.rank) a.rank[at] = in ? rank : -1;
}
__device__ __forceinline__ void write_top(const LogprobArgs& a, size_t at, const RowSums& r, u64 key) {
  if (a.top_logprob) a.top_logprob[at] = r.logprob(key_value((unsigned)(key >> 32)));
  if (a.top_token) a.top_token[at] = (int)~(unsigned)key;
}

// One workgroup per row and chunk.  PARTS: the chunk's share goes to the workspace.
template <int TYPE, int W, bool PARTS>
__global__ __launch_bounds__(W * 64) void k_logprobs(LogprobArgs a, Parts parts, int chunks) {
  using L = Logit<TYPE>;
  constexpr int VE = 16 / L::size, NV = kLpVals / VE, TH = W * 64;
  __shared__ float s_m[W], s_S[W], s_T[W];
  __shared__ unsigned s_key[W];
  __shared__ int s_count[W][kLpTokens];
  __shared__ u64 s_list[kLpList], s_best[W];
  __shared__ int s_n;
  const int r = PARTS ? blockIdx.x / chunks : blockIdx.x, chunk = PARTS ? blockIdx.x % chunks : 0;
  const int V = a.vocab, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint8_t* row = (const uint8_t*)a.x + (size_t)r * a.stride * L::size;
  // 16-byte blocks from the one that holds the row's first logit, which is its
  // element `skew`; a block that is not the row's alone is read by elements
  const int skew = (int)(((uintptr_t)row & 15) / L::size);
  const uint8_t* first = row - skew * L::size;
  const int b0 = chunk * (TH * NV) + tid;
  float x[kLpVals];
  auto token = [&](int i) { return (b0 + i / VE * TH) * VE + i % VE - skew; };  // token of x[i]
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int t0 = token(v * VE);
    if (t0 >= 0 && t0 + VE <= V) {
      L::spread(*(const uint4*)(first + (size_t)(b0 + v * TH) * 16), x + v * VE);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) x[v * VE + e] = t0 + e >= 0 && t0 + e < V ? L::at(row, t0 + e) : -INFINITY;
    }
  }
  float xt[kLpTokens];
  int tok[kLpTokens];
#pragma unroll
  for (int t = 0; t < kLpTokens; ++t)
    if (t < a.n_tokens) {
      tok[t] = a.tokens[(size_t)r * a.n_tokens + t];
      xt[t] = tok[t] >= 0 && tok[t] < V ? L::at(row, tok[t]) : 0.f;
    }
  if (tid == 0) s_n = 0;

  float lm = x[0];
#pragma unroll
  for (int i = 1; i < kLpVals; ++i) lm = fmaxf(lm, x[i]);
  lm = lm != lm ? -INFINITY : lm;
  const float wm = wave_reduce(lm, [](float p, float q) { return fmaxf(p, q); });
  unsigned cut = 0;
  if (a.top_k > 0) {
    const unsigned k = order_key(lm);
    const int need = (a.top_k + W - 1) / W;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
      const unsigned c = cut | (1u << bit);
      cut = __popcll(__ballot(k >= c)) >= need ? c : cut;
    }
  }
  if (lane == 0) {
    s_m[wave] = wm;
    s_key[wave] = cut;
  }
  __syncthreads();
  RowSums rs;
  rs.m = s_m[0];
  cut = s_key[0];
#pragma unroll
  for (int w = 1; w < W; ++w) {
    rs.m = fmaxf(rs.m, s_m[w]);
    cut = min(cut, s_key[w]);
  }
  const float base = rs.base();

  float S = 0.f, T = 0.f;
#pragma unroll
  for (int i = 0; i < kLpVals; ++i) {
    const float d = x[i] - base, e = __builtin_amdgcn_exp2f(d * kLog2e);
    S += e;
    T += e * fmaxf(d, -1e30f);  // d = -inf has e = 0
  }
  S = wave_reduce(S, [](float p, float q) { return p + q; });
  T = wave_reduce(T, [](float p, float q) { return p + q; });
#pragma unroll
  for (int t = 0; t < kLpTokens; ++t)
    if (t < a.n_tokens) {
      int n = 0;
      const float y = xt[t];
      u64 equal = 0;
      if (y == y) {
#pragma unroll
        for (int i = 0; i < kLpVals; ++i) {
          n += __popcll(__ballot(!(x[i] <= y)));
          equal |= __ballot(x[i] == y);
        }
      } else {
        equal = ~0ull;
      }
      if (equal) {
#pragma unroll
        for (int i = 0; i < kLpVals; ++i) {
          const int k = token(i);
          n += __popcll(__ballot((x[i] == y || (x[i] != x[i] && y != y)) && k >= 0 && k < tok[t]));
        }
      }
      if (lane == 0) s_count[wave][t] = n;
    }
  if (lane == 0) {
    s_S[wave] = S;
    s_T[wave] = T;
  }
  if (a.top_k > 0) {
    // everything at or above the cut; where the cut is at -inf, of the logits
    // of -inf only the chunk's first top_k tokens
    const float c = cut > order_key(-INFINITY) ? key_value(cut) : -INFINITY;
    const int early = max(0, chunk * (TH * NV) * VE - skew) + a.top_k;
#pragma unroll
    for (int i = 0; i < kLpVals; ++i) {
      if (!(x[i] < c)) {
        const int k = token(i);
        if (x[i] != -INFINITY || (k >= 0 && k < V && k < early)) {
          const int at = atomicAdd(&s_n, 1);
          if (at < kLpList) s_list[at] = pair_key(x[i], k);
        }
      }
    }
  }
  __syncthreads();
  rs.S = s_S[0];
  rs.T = s_T[0];
#pragma unroll
  for (int w = 1; w < W; ++w) {
    rs.S += s_S[w];
    rs.T += s_T[w];
  }
  const size_t part = blockIdx.x;
  if (tid < a.n_tokens) {
    int n = 0;
    for (int w = 0; w < W; ++w) n += s_count[w][tid];
    if constexpr (PARTS) {
      parts.counts[part * a.n_tokens + tid] = n;
    } else {
      const size_t at = (size_t)r * a.n_tokens + tid;
      const int k = a.tokens[at];
      write_token(a, at, rs, k, k >= 0 && k < V ? L::at(row, k) : 0.f, n);
    }
  }
  if (tid == 0) {
    if constexpr (PARTS) {
      parts.sums[part * 3] = rs.m;
      parts.sums[part * 3 + 1] = rs.S;
      parts.sums[part * 3 + 2] = rs.T;
    } else if (a.entropy) {
      a.entropy[r] = rs.entropy();
    }
  }
  if (a.top_k == 0) return;
  auto put = [&](int place, u64 key) {
    if constexpr (PARTS)
      parts.keys[part * a.top_k + place] = key;
    else
      write_top(a, (size_t)r * a.top_k + place, rs, key);
  };
  const int n = s_n;
  if (n <= kLpList) {
    for (int i = tid; i < n; i += TH) {
      const u64 k = s_list[i];
      int place = 0;
      for (int j = 0; j < n; ++j) place += s_list[j] > k;
      if (place < a.top_k) put(place, k);
    }
    for (int i = n + tid; i < a.top_k; i += TH) put(i, 0);
    return;
  }
  // one by one: every thread's largest key below those taken, the largest of them
  u64 mine = 0, taken = ~0ull;
  bool stale = true;
  for (int t = 0; t < a.top_k; ++t) {
    if (stale) {
      mine = 0;
#pragma unroll
      for (int i = 0; i < kLpVals; ++i) {
        const int tk = token(i);
        const u64 k = tk >= 0 && tk < V ? pair_key(x[i], tk) : 0;
        if (k < taken && k > mine) mine = k;
      }
    }
    const u64 best = wave_reduce(mine, [](u64 p, u64 q) { return p > q ? p : q; });
    __syncthreads();
    if (lane == 0) s_best[wave] = best;
    __syncthreads();
    taken = s_best[0];
#pragma unroll
    for (int w = 1; w < W; ++w) taken = s_best[w] > taken ? s_best[w] : taken;
    stale = mine == taken;
    if (tid == 0) put(t, taken);
  }
}

// Joins a row's chunks; one workgroup per row.
template <int TYPE>
__global__ __launch_bounds__(256) void k_logprobs_join(LogprobArgs a, Parts parts, int chunks) {
  using L = Logit<TYPE>;
  const int r = blockIdx.x, tid = threadIdx.x, k = a.top_k;
  extern __shared__ u64 keys[];  // [chunks][k]
  const size_t part = (size_t)r * chunks;
  for (int i = tid; i < chunks * k; i += 256) keys[i] = parts.keys[part * k + i];
  // every thread sums all chunks, in their order
  RowSums rs{-INFINITY, 0.f, 0.f};
  for (int c = 0; c < chunks; ++c) rs.m = fmaxf(rs.m, parts.sums[(part + c) * 3]);
  const float base = rs.base();
  for (int c = 0; c < chunks; ++c) {
    const float* p = parts.sums + (part + c) * 3;
    if (p[0] == -INFINITY) {
      rs.S += p[1];  // 0, or NaN
      continue;
    }
    const float d = p[0] - base, f = expf(d);
    rs.S += p[1] * f;
    rs.T += f == 0.f ? 0.f : f * (p[2] + d * p[1]);
  }
  if (tid == 0 && a.entropy) a.entropy[r] = rs.entropy();
  if (tid < a.n_tokens) {
    int n = 0;
    for (int c = 0; c < chunks; ++c) n += parts.counts[(part + c) * a.n_tokens + tid];
    const size_t at = (size_t)r * a.n_tokens + tid;
    const int tok = a.tokens[at];
    const void* row = (const uint8_t*)a.x + (size_t)r * a.stride * L::size;
    write_token(a, at, rs, tok, tok >= 0 && tok < a.vocab ? L::at(row, tok) : 0.f, n);
  }
  __syncthreads();
  // a key's place: its place in its own chunk, and the keys before it in the
  // others, whose lists are in order
  for (int i = tid; i < chunks * k; i += 256) {
    const u64 key = keys[i];
    const int own = i / k;
    int place = i % k;
    for (int c = 0; c < chunks && place < k; ++c) {
      if (c == own) continue;
      int lo = 0, hi = k;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (keys[c * k + mid] > key)
          lo = mid + 1;
        else
          hi = mid;
      }
      place += lo;
    }
    if (key != 0 && place < k) write_top(a, (size_t)r * k + place, rs, key);
  }
}

// Chunks of a row: none where a workgroup of up to 1024 threads holds it all
// (the launch then writes the results itself), else of 256 threads.  A row may
// start inside a 16-byte block.
struct Plan {
  int waves, chunks;
};
Plan plan(int vocab) {
  const int most = vocab + 7;
  for (int w = 4; w <= 16; w *= 2)
    if (most <= w * 64 * kLpVals) return {w, 1};
  return {4, (most + 4 * 64 * kLpVals - 1) / (4 * 64 * kLpVals)};
}

size_t align16(size_t n) { return (n + 15) & ~(size_t)15; }

}  // namespace

bool logprobs_fit(int rows, int vocab) {
  return vocab <= kLogprobVocab && (int64_t)rows * plan(vocab).chunks <= (1 << 22);
}

size_t logprobs_bytes(int rows, int vocab, int n_tokens, int top_k) {
  const size_t c = (size_t)plan(vocab).chunks * rows;
  if (plan(vocab).chunks == 1) return 0;
  return align16(c * 12) + align16(c * n_tokens * 4) + c * top_k * 8;
}

template <int TYPE>
static hipError_t launch_typed(const LogprobArgs& a, uint8_t* ws, hipStream_t s) {
  const Plan p = plan(a.vocab);
  Parts parts{};
  const dim3 grid(p.chunks * a.rows);
  if (p.chunks > 1) {
    const size_t c = (size_t)p.chunks * a.rows;
    parts.sums = (float*)ws;
    parts.counts = (int*)(ws + align16(c * 12));
    parts.keys = (u64*)(ws + align16(c * 12) + align16(c * a.n_tokens * 4));
    TSS_LAUNCH((k_logprobs<TYPE, 4, true>), grid, dim3(256), 0, s, a, parts, p.chunks);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    TSS_LAUNCH(k_logprobs_join<TYPE>, dim3(a.rows), dim3(256), (size_t)p.chunks * a.top_k * 8, s, a, parts, p.chunks);
  } else if (p.waves == 4) {
    TSS_LAUNCH((k_logprobs<TYPE, 4, false>), grid, dim3(256), 0, s, a, parts, p.chunks);
  } else if (p.waves == 8) {
    TSS_LAUNCH((k_logprobs<TYPE, 8, false>), grid, dim3(512), 0, s, a, parts, p.chunks);
  } else {
    TSS_LAUNCH((k_logprobs<TYPE, 16, false>), grid, dim3(1024), 0, s, a, parts, p.chunks);
  }
  return hipGetLastError();
}

hipError_t launch_logprobs(const LogprobArgs& a, void* ws, hipStream_t s) {
  if (a.rows < 1 || a.vocab < 1) return hipErrorInvalidValue;
  if (a.type == TSS_T_F32) return launch_typed<TSS_T_F32>(a, (uint8_t*)ws, s);
  if (a.type == TSS_T_F16) return launch_typed<TSS_T_F16>(a, (uint8_t*)ws, s);
  return launch_typed<TSS_T_BF16>(a, (uint8_t*)ws, s);
}

}  // namespace tss
