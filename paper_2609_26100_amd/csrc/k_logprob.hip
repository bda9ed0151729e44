// Log probabilities of given tokens, entropy and alternatives (gfx950).
//
// With m = max x, S = sum e^(x - m) and T = sum (x - m) e^(x - m) of a row:
//   logprob = x - m - ln S,  entropy = ln S - T / S.
//
// A workgroup takes a chunk of a row, 32 logits a thread, into registers with
// 16-byte loads, so HBM is read once, and goes over the registers twice: for
// the maxima, and for S, T, the ranks and the candidates of the alternatives.
//   * Ranks: a token's rank is the number of logits that come before it: the sign
//     of a difference each (a compare's mask in a scalar register would make the
//     next instruction wait), skipped where no logit of the wave reaches the token's.
//   * Alternatives: the k-th largest of the threads' maxima (its top 16 bits) has
//     at least k logits at or above it, and few more, and only threads whose maximum
//     reaches it hold any.  Each of W waves finds the ceil(k / W)-th largest of its
//     share by bisection over ballots, and the least of these is the cut.  The
//     threads that reach it are listed, all threads look through their logits, and
//     what is found goes to a list in LDS, where each counts how many precede it.
//     Keys of (logit, token) are unique, so the order in which they got there does
//     not matter.  Where too many are equal for the list, the cut is made finer, 8
//     bits of the key at a time.
// Rows of more than one chunk leave (m, S, T), counts and the top 16 bits of every
// thread's maximum (2 bytes for 32 logits) for each chunk in the workspace, and a
// second launch joins them: the alternatives are looked for once a row, not once a
// chunk (20 of 2048 rows of 131072 bf16 take 21 us more than none; looked for in
// every chunk they took 66).
//
// Bound by HBM for many rows without tokens or alternatives (2048 rows of 131072
// bf16, 537 MB: 100 us, 5.4 TB/s); a token's rank adds two instructions a logit
// (+ 30 us there, less for a likely token, whose chunks are mostly skipped).
#include "../../include/tss.h"
#include "tss_internal.h"

#include <type_traits>

namespace tss {

namespace {

constexpr int kLpVals = 32;       // logits a thread holds
constexpr int kLpList = 512;      // candidates in LDS
constexpr int kLpHolders = 256;   // threads that are looked through
constexpr int kLpTokens = TSS_LOGPROBS_MAX_TOKENS;
constexpr float kLpFar = 65536.f; // maxima beyond it take the logits' differences first
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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

// The same value, of which the compiler does not know it: what a rare path
// computes again from it is not kept in registers from the first time.
__device__ __forceinline__ float again(float x) {
  asm volatile("" : "+v"(x));
  return x;
}

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
// bits shifted up by one, the sign of d below them.
__device__ __forceinline__ unsigned push_sign(unsigned bits, float d) {
  return __builtin_amdgcn_alignbit(bits, __float_as_uint(d), 31);
}

// What a row's (m, S, T) and a token's logit come to.
struct RowSums {
  float m, S, T;
  __device__ float base() const { return m == -INFINITY ? 0.f : m; }
  // a row without a token left has nothing to share out
  __device__ float logprob(float x) const { return S == 0.f ? -INFINITY : x - base() - logf(S); }
  __device__ float entropy() const { return S == 0.f ? 0.f : logf(S) - T / S; }
};

// The chunks' shares of the rows in the workspace (row-major over rows and chunks).
struct Parts {
  float* sums;      // [rows * chunks][3]: m, S, T
  int* counts;      // [rows * chunks][n_tokens]
  uint16_t* tops;   // [rows * chunks][256]: top 16 bits of the key of each thread's maximum
};

// Shared by the threads that look for a row's alternatives.
struct Search {
  __align__(16) u64 list[kLpList];
  int n, holders, bins[256], bin, above;
  unsigned cut[16];
  int holder[kLpHolders];
};

// The first k logits of a row of `tokens`, by W waves.  mine: the largest key (its top 16 bits) of
// a share of the logits; the threads of the first `waves` waves all have some.
// holders(cut, hold): calls hold(id) for the threads of the first launch that it knows to reach the
// cut; logits(id, i, f): f(logit, token) for logit i < kLpVals of such a thread, if there is one;
// each(f): f(logit, token) for this thread's share of the row; one(token): its logit.  All
// threads call it.
template <typename Holders, typename Logits, typename Each, typename One, typename Put>
__device__ __forceinline__ void find_top(Search& s, int k, int tokens, unsigned mine, int W, int waves, Holders holders,
                                         Logits logits, Each each, One one, Put put) {
  const int tid = threadIdx.x, TH = W * 64, wave = tid >> 6;
  for (int i = tid; i < kLpList; i += TH) s.list[i] = 0;
  if (tid == 0) s.n = s.holders = 0;
  unsigned cut = 0;
  const int need = (k + waves - 1) / waves;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const unsigned c = cut | (1u << bit);
    cut = __popcll(__ballot(mine >= c)) >= need ? c : cut;
  }
  if ((tid & 63) == 0) s.cut[wave] = wave < waves ? cut : 0xffffu;
  __syncthreads();
  cut = s.cut[0];
  for (int w = 1; w < W; ++w) cut = min(cut, s.cut[w]);
  auto list = [&](float z, int t) {
    const int at = atomicAdd(&s.n, 1);
    if (at < kLpList) s.list[at] = pair_key(z, t);
  };
  // a cut at -inf: of the logits of -inf only those of the first k tokens
  const unsigned none = order_key(-INFINITY);
  const bool low = cut <= none >> 16;
  const unsigned least = low ? none + 1 : cut << 16;
  if (low && tid < k && tid < tokens && one(tid) == -INFINITY) list(-INFINITY, tid);
  holders(low ? least >> 16 : cut, [&](int id) {
    const int at = atomicAdd(&s.holders, 1);
    if (at < kLpHolders) s.holder[at] = id;
  });
  __syncthreads();
  const bool few = s.holders <= kLpHolders;
  if (few) {
    for (int i = tid; i < s.holders * kLpVals; i += TH)
      logits(s.holder[i / kLpVals], i % kLpVals, [&](float z, int t) {
        if (order_key(z) >= least) list(z, t);
      });
    __syncthreads();
  }
  if (!few || s.n > kLpList) {
    // finer: the least prefix of the keys, 8 bits longer each time, that at least k keys reach
    __syncthreads();
    u64 prefix = 0;
    int above = 0;  // keys beyond the prefix's
    for (int shift = 56; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += TH) s.bins[i] = 0;
      __syncthreads();
      each([&](float z, int t) {
        const u64 key = pair_key(z, t);
        if (shift == 56 || key >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&s.bins[(key >> shift) & 255], 1);
      });
      __syncthreads();
      if (tid == 0) {
        int b = 255, over = above;
        while (b > 0 && over + s.bins[b] < k) over += s.bins[b--];
        s.bin = b;
        s.above = over;
      }
      __syncthreads();
      above = s.above;
      prefix |= (u64)s.bin << shift;
      const int reach = above + s.bins[s.bin];
      __syncthreads();
      if (reach <= kLpList) break;
    }
    if (tid == 0) s.n = 0;
    for (int i = tid; i < kLpList; i += TH) s.list[i] = 0;
    __syncthreads();
    each([&](float z, int t) {
      if (pair_key(z, t) >= prefix) list(z, t);
    });
    __syncthreads();
  }
  const int n = min(s.n, kLpList);
  for (int i = tid; i < n; i += TH) {
    const u64 key = s.list[i];
    int place = 0;
    for (int j = 0; j < n; j += 8) {  // zeros behind the last
#pragma unroll
      for (int u = 0; u < 8; ++u) place += s.list[j + u] > key;
    }
    if (place < k) put(place, key);
  }
}

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

// grid (rows, chunks).  PARTS: the chunk's share goes to the workspace.
template <int TYPE, int W, bool PARTS>
__global__ __launch_bounds__(W * 64, PARTS ? 6 : 1) void k_logprobs(LogprobArgs a, Parts parts, int chunks) {
  using L = Logit<TYPE>;
  constexpr int VE = 16 / L::size, NV = kLpVals / VE, TH = W * 64;
  __shared__ float s_m[W], s_S[W], s_T[W];
  __shared__ int s_count[W][kLpTokens];
  const int r = blockIdx.x, chunk = PARTS ? blockIdx.y : 0;
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
  const int c0 = chunk * (TH * NV) * VE - skew;  // the chunk's first token
  uint4 raw[NV];
  if (c0 >= 0 && c0 + TH * kLpVals <= V) {
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v] = *(const uint4*)(first + (unsigned)(b0 + v * TH) * 16u);
#pragma unroll
    for (int v = 0; v < NV; ++v) L::spread(raw[v], x + v * VE);
  } else {
    // the row's first and last chunk: what lies outside is -inf
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int t0 = token(v * VE);
      raw[v] = uint4{0, 0, 0, 0};
      if (t0 >= 0 && t0 + VE <= V) raw[v] = *(const uint4*)(first + (unsigned)(b0 + v * TH) * 16u);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int t0 = token(v * VE);
      L::spread(raw[v], x + v * VE);
      if (t0 < 0 || t0 + VE > V) {
#pragma unroll
        for (int e = 0; e < VE; ++e) x[v * VE + e] = t0 + e >= 0 && t0 + e < V ? L::at(row, t0 + e) : -INFINITY;
      }
    }
  }
  // what the rare paths read: the thread's logits from the cache again, so that
  // they take no registers from the common ones
  auto each = [&](auto f) {
#pragma unroll 8
    for (int i = 0; i < kLpVals; ++i) {
      const int k = token(i);
      if (k >= 0 && k < V) f(L::at(row, k), k);
    }
  };
  // lane t of every wave has given token t and its logit; a token outside the
  // vocabulary is -1 from here on and is looked for nowhere
  int tok = -1;
  float xt = 0.f;
  if (lane < a.n_tokens) {
    tok = a.tokens[(size_t)r * a.n_tokens + lane];
    if (tok < 0 || tok >= V) tok = -1;
    if (tok >= 0) xt = L::at(row, tok);
  }

  float lm = x[0];
#pragma unroll
  for (int i = 1; i < kLpVals; ++i) lm = fmaxf(lm, x[i]);
  lm = lm != lm ? -INFINITY : lm;
  const float wm = wave_max(lm);
  if (lane == 0) s_m[wave] = wm;
  __syncthreads();
  RowSums rs;
  rs.m = s_m[0];
#pragma unroll
  for (int w = 1; w < W; ++w) rs.m = fmaxf(rs.m, s_m[w]);
  const float base = rs.base();

  // (x - m) log2 e as one fma: the rounding of m log2 e shifts all of them by
  // the same `shift`, which is taken out of the sums again (up to kLpFar it is at most
  // 2^-8; the shift of a maximum of 1e10 would be hundreds of powers of two)
  const float b2 = base * kLog2e, shift = fmaf(base, kLog2e, -b2);
  float S = 0.f, T = 0.f;
#pragma unroll
  for (int i = 0; i < kLpVals; ++i) {
    const float d = fmaf(x[i], kLog2e, -b2), e = __builtin_amdgcn_exp2f(d);
    S += e;
    T = fmaf(e, d, T);
  }
  if (fabsf(base) > kLpFar) {  // subtracted first, in two instructions a logit
    S = T = 0.f;
    const float base2 = again(base);
#pragma unroll
    for (int i = 0; i < kLpVals; ++i) {
      const float d = x[i] - base2, e = __builtin_amdgcn_exp2f(d * kLog2e);
      S += e;
      T = e == 0.f ? T : fmaf(e, d, T);
    }
  } else {
    if (__any(T != T)) {  // logits of -inf have e = 0 (where it is not NaN for good)
      T = 0.f;
      const float b3 = again(b2);
#pragma unroll
      for (int i = 0; i < kLpVals; ++i) {
        const float d = fmaf(x[i], kLog2e, -b3), e = __builtin_amdgcn_exp2f(d);
        T = e == 0.f ? T : fmaf(e, d, T);
      }
    }
    const float f = __builtin_amdgcn_exp2f(-shift);
    T = (T - shift * S) * f * kLn2;
    S *= f;
  }
  const float lane_S = S;
  S = wave_sum(S);
  T = wave_sum(T);
  // A logit is less than c where the sign of x - c is set (c = 0 taken as -0).
  // That is not so for NaN and between infinities, which leave a lane's sum NaN.
  const bool odd = __any(lane_S != lane_S);
  for (int t = 0; t < a.n_tokens; ++t) {
    int n = 0;
    const float y = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(xt), t));
    const int at = __builtin_amdgcn_readlane(tok, t);
    if (at < 0 || (wm < y && !odd)) {
      // no such token (its rank is -1), or nothing of this wave's comes before it
    } else if (fabsf(y) < INFINITY && !odd) {
      // before the token an equal logit counts, behind it only a larger one:
      // at least y, or at least the float after it
      const float up = y == 0.f ? __uint_as_float(1u) : __uint_as_float(__float_as_uint(y) + (y > 0.f ? 1u : -1u));
      if (at < c0 || at >= c0 + TH * kLpVals) {
        const float c = at < c0 ? up : y == 0.f ? -0.f : y;
        unsigned less = 0;
#pragma unroll
        for (int i = 0; i < kLpVals; ++i) less = push_sign(less, x[i] - c);
        n = kLpVals - __popc(less);
      } else {  // the row's chunk that holds the token; its block counts as behind it at first
        unsigned less = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int t0 = token(v * VE);
          const float c = t0 + VE <= at ? (y == 0.f ? -0.f : y) : up;
#pragma unroll
          for (int e = 0; e < VE; ++e) less = push_sign(less, x[v * VE + e] - c);
        }
        n = kLpVals - __popc(less);
        const int blk = (at + skew) / VE;  // the thread that has it looks again at what stands before it
        if (blk % TH == tid)
          for (int k = max(0, blk * VE - skew); k < at; ++k) n += L::at(row, k) == y;
      }
    } else {
      each([&](float z, int k) { n += pair_key(z, k) > pair_key(y, at); });
    }
    n = wave_sum(n);
    if (lane == 0) s_count[wave][t] = n;
  }
  if (lane == 0) {
    s_S[wave] = S;
    s_T[wave] = T;
  }
  __syncthreads();
  rs.S = s_S[0];
  rs.T = s_T[0];
#pragma unroll
  for (int w = 1; w < W; ++w) {
    rs.S += s_S[w];
    rs.T += s_T[w];
  }
  const size_t part = (size_t)r * chunks + chunk;
  if (tid < a.n_tokens) {
    int n = 0;
    for (int w = 0; w < W; ++w) n += s_count[w][tid];
    if constexpr (PARTS) {
      parts.counts[part * a.n_tokens + tid] = n;
    } else {
      write_token(a, (size_t)r * a.n_tokens + tid, rs, tok, xt, n);
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
  unsigned top = order_key(lm) >> 16;
  if (odd) {  // NaN orders as the largest (infinities leave NaN in the sums as well)
    bool nan = false;
    each([&](float z, int) { nan |= z != z; });
    if (nan) top = 0xffffu;
  }
  if constexpr (PARTS) {
    static_assert(TH == 256, "as Parts has it");
    parts.tops[part * TH + tid] = (uint16_t)top;
  } else {
    __shared__ Search s;
    auto get = [&](int id, int i, auto f) {
      const int k = (id + i / VE * TH) * VE + i % VE - skew;
      if (k >= 0 && k < V) f(L::at(row, k), k);
    };
    auto all = [&](auto f) {
#pragma unroll 8
      for (int i = 0; i < kLpVals; ++i) get(tid, i, f);
    };
    // waves whose threads all have some of the row (at least the first)
    const int waves = max(1, min(W, (V + skew) / VE / 64));
    find_top(s, a.top_k, V, top, W, waves,
             [&](unsigned cut, auto hold) {
               if (top >= cut) hold(tid);
             },
             get, all, [&](int t) { return L::at(row, t); },
             [&](int place, u64 key) { write_top(a, (size_t)r * a.top_k + place, rs, key); });
  }
}

// sum (x - to) e^(x - to) of terms with sums S and T = sum (x - m) e^(x - m),
// f = e^(m - to); 0 for terms that vanish, and for none (m = -inf, f = 1).
__device__ __forceinline__ float shifted(float S, float T, float f, float m, float to) {
  return f == 0.f || m == -INFINITY ? 0.f : f * (T + (m - to) * S);
}

// Joins a row's chunks; one workgroup per row.
template <int TYPE>
__global__ __launch_bounds__(256) void k_logprobs_join(LogprobArgs a, Parts parts, int chunks) {
  using L = Logit<TYPE>;
  const int r = blockIdx.x, tid = threadIdx.x, k = a.top_k;
  const size_t part = (size_t)r * chunks;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  __shared__ Search s;
  constexpr int VE = 16 / L::size, TH = 256, NV = kLpVals / VE;
  const int V = a.vocab;
  const uint8_t* row = (const uint8_t*)a.x + (size_t)r * a.stride * L::size;
  const int skew = (int)(((uintptr_t)row & 15) / L::size);
  // thread h of chunk c is id c * 256 + h; a thread here has eight next to each other at a time
  const uint4* tops = (const uint4*)(parts.tops + part * TH);
  auto eights = [&](auto f) {
    for (int i = tid; i < chunks * TH / 8; i += 256) {
      const uint4 t = tops[i];
      const unsigned w[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
      for (int u = 0; u < 8; ++u) f(i * 8 + u, u & 1 ? w[u >> 1] >> 16 : w[u >> 1] & 0xffffu);
    }
  };
  unsigned top = 0;
  if (k > 0) eights([&](int, unsigned t) { top = max(top, t); });
  int tok = -1;
  float xt = 0.f;
  if (lane < a.n_tokens) {
    tok = a.tokens[(size_t)r * a.n_tokens + lane];
    if (tok >= 0 && tok < a.vocab) xt = L::at((const uint8_t*)a.x + (size_t)r * a.stride * L::size, tok);
  }
  // every wave sums all chunks, a lane each
  float m = -INFINITY, S = 0.f, T = 0.f;
  for (int c = lane; c < chunks; c += 64) {
    const float* p = parts.sums + (part + c) * 3;
    const RowSums one{p[0], p[1], p[2]};
    const float top = fmaxf(m, one.m), to = top == -INFINITY ? 0.f : top;
    const float f = m == -INFINITY ? 1.f : expf(m - to), g = one.m == -INFINITY ? 1.f : expf(one.m - to);
    T = shifted(S, T, f, m, to) + shifted(one.S, one.T, g, one.m, to);
    S = S * f + one.S * g;
    m = top;
  }
  RowSums rs;
  rs.m = wave_max(m);
  const float base = rs.base(), f = m == -INFINITY ? 1.f : expf(m - base);
  rs.T = wave_sum(shifted(S, T, f, m, base));
  rs.S = wave_sum(S * f);
  if (tid == 0 && a.entropy) a.entropy[r] = rs.entropy();
  for (int t = wave; t < a.n_tokens; t += 4) {
    int n = 0;
    for (int c = lane; c < chunks; c += 64) n += parts.counts[(part + c) * a.n_tokens + t];
    n = wave_sum(n);
    if (lane == t) write_token(a, (size_t)r * a.n_tokens + t, rs, tok, xt, n);
  }
  if (k == 0) return;
  auto get = [&](int id, int i, auto f) {
    const int t = (id / TH * (TH * NV) + id % TH + i / VE * TH) * VE + i % VE - skew;
    if (t >= 0 && t < V) f(L::at(row, t), t);
  };
  auto all = [&](auto f) {
#pragma unroll 8
    for (int t = tid; t < V; t += 256) f(L::at(row, t), t);
  };
  find_top(s, k, V, top, 4, max(1, min(4, chunks / 2)),
           [&](unsigned cut, auto hold) {
             eights([&](int id, unsigned t) {
               if (t >= cut) hold(id);
             });
           },
           get, all, [&](int t) { return L::at(row, t); },
           [&](int place, u64 key) { write_top(a, (size_t)r * k + place, rs, key); });
}

// Chunks of a row: one where a workgroup of up to 1024 threads holds it all (the
// launch then writes the results itself), else of 256 threads.  skew: logits
// that may stand before the row's first in its 16-byte block (7 at most).
struct Plan {
  int waves, chunks;
};
Plan plan(int vocab, int skew) {
  const int most = vocab + skew;
  for (int w = 4; w <= 16; w *= 2)
    if (most <= w * 64 * kLpVals) return {w, 1};
  return {4, (most + 4 * 64 * kLpVals - 1) / (4 * 64 * kLpVals)};
}

size_t align16(size_t n) { return (n + 15) & ~(size_t)15; }

}  // namespace

bool logprobs_fit(int rows, int vocab) {
  return vocab <= kLogprobVocab && (int64_t)rows * plan(vocab, 7).chunks <= (1 << 22);
}

size_t logprobs_bytes(int rows, int vocab, int n_tokens, int top_k) {
  const size_t chunks = plan(vocab, 7).chunks, c = chunks * rows;
  if (chunks == 1) return 0;
  return align16(c * 12) + align16(c * n_tokens * 4) + (top_k > 0 ? c * 512 : 0);
}

template <int TYPE>
static hipError_t launch_typed(const LogprobArgs& a, uint8_t* ws, hipStream_t s) {
  constexpr int ES = Logit<TYPE>::size;
  const bool blocks = (uintptr_t)a.x % 16 == 0 && (a.rows == 1 || a.stride * ES % 16 == 0);
  const Plan p = plan(a.vocab, blocks ? 0 : 16 / ES - 1);
  Parts parts{};
  const dim3 grid(a.rows, p.chunks);
  if (p.chunks > 1) {
    const size_t c = (size_t)p.chunks * a.rows;
    parts.sums = (float*)ws;
    parts.counts = (int*)(ws + align16(c * 12));
    parts.tops = (uint16_t*)(ws + align16(c * 12) + align16(c * a.n_tokens * 4));
    TSS_LAUNCH((k_logprobs<TYPE, 4, true>), grid, dim3(256), 0, s, a, parts, p.chunks);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    TSS_LAUNCH(k_logprobs_join<TYPE>, dim3(a.rows), dim3(256), 0, s, a, parts, p.chunks);
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
