// The n best continuations of each group of beams (gfx950).
//
// A candidate (beam b, token t) is worth scores[b] + x[b][t] - ln sum e^x[b].
//
// The first launch reads the logits once: a wave takes 2048 of a row ("part"), 32 a lane,
// and leaves the part's maximum m and S = sum e^(x - m), and every lane's largest logit
// (in the logits' type, so exactly; 3 % of the bytes read).  Waves meet nowhere.
//
// The second has a workgroup for each group.  It joins the rows' sums and finds a cut that
// at least n candidates reach: every thread has the best of its share of the parts of the beams
// that can win (of their lanes, where parts are few), and the n-th best thread is the cut (found
// among those that reach the lowest of the waves' own cuts, a bisection over ballots each).
// Then it opens what reaches the cut, parts, lanes, logits, and the few candidates found (38
// for n = 32) are ordered by counting how many precede each.  Where the best candidates are in
// few of the parts, a second cut is found among the lanes of the parts that reach the first.
// Where too many are equal for the lists, the cut is searched for bit by bit over all logits of
// the group (16 beams of 32000 equal logits 1.3 ms).
//
// Bound by HBM where there is much to read (32 groups of 16 beams of 131072 bf16 logits, 134 MB:
// the first launch 24 us, 5.6 TB/s; the second 13.5, on 32 CUs), else by the dependent
// phases of two launches (four beams of 32000 fp32: 3.8 + 8.3 us, of which the second's
// sums take 1.6, its cut 3, what is opened 2.1 and the order 0.7).
//
// Values are (x - m) + c in 64 bits, c the score less the logarithm.  In S, 8 exponentials
// are summed in fp32 and the rest in 64 bits: a logarithm is off by the rounding of the
// exponents' arguments and by the exponentials' own, 3e-8 in the mean of squares and up to
// 2e-7 over rows of 1000 to 131072 normal logits, where scores of -10 have steps of 1e-6.
// Equal rows have equal sums wherever they begin, so that their candidates are ties.
#include "logits.h"

namespace tss {

namespace {

constexpr int kBeamVals = 32;                    // logits of a lane
constexpr int kBeamPart = 64 * kBeamVals;        // of a part
constexpr int kBeamWaves = 4;                    // parts of a workgroup
constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64;
constexpr int kPickList = 1024;                  // candidates, opened parts
constexpr int kPickHolders = 2048;               // opened lanes
// Parts that beams must have for each candidate, else their lanes are looked through at once.  With
// 1 one of 32 beams of 131072 tokens, n = 64, takes 34.5 us a call in a graph, with 2 and 4 27.9;
// with 4 one of 16 beams of 200000, n = 32, 27.2, with 1 and 2 23.0.
constexpr int kPickParts = 2;
// Lanes that reach the parts' cut beyond which another is found.  With 512, four beams of 32000 masked
// down to 1500 tokens each take 97 us, with 256 21; with 1024, 32 beams of 20000 whose scores are 1.5
// apart 351, with 256 and 512 34.
constexpr int kPickMany = 256;
constexpr double kNoCut = -1.7976931348623157e308;  // every candidate reaches it
constexpr double kLog2eD = 1.4426950408889634074;
constexpr float kLog2eHi = (float)kLog2eD, kLog2eLo = (float)(kLog2eD - (double)kLog2eHi);

typedef unsigned long long u64;

// What the first launch leaves, row-major over rows and parts.
struct BeamParts {
  double* sums;      // [rows * parts]
  float* tops;       // [rows * parts] part's largest logit
  void* lanes;       // [rows * parts][64] lane's largest logit, in the logits' type
};

// 16 bytes of a row, from any element on.
typedef unsigned Raw __attribute__((ext_vector_type(4), aligned(2)));

template <int TYPE>
__device__ __forceinline__ const uint8_t* row_at(const BeamArgs& a, int r) {
  return (const uint8_t*)a.x + (size_t)r * a.stride * Logit<TYPE>::size;
}

// Token of element i of lane l of a part.
template <int TYPE>
__device__ __forceinline__ int token_of(int part, int l, int i) {
  constexpr int VE = 16 / Logit<TYPE>::size;
  return ((part * (kBeamVals / VE) + i / VE) * 64 + l) * VE + i % VE;
}

template <int TYPE>
__device__ __forceinline__ void store_top(void* to, size_t at, float x) {
  if constexpr (TYPE == TSS_T_F32) ((float*)to)[at] = x;
  if constexpr (TYPE == TSS_T_F16) ((_Float16*)to)[at] = (_Float16)x;
  if constexpr (TYPE == TSS_T_BF16) ((uint16_t*)to)[at] = (uint16_t)(__float_as_uint(x) >> 16);
}

__device__ __forceinline__ double sum64(double x) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
  return x;
}

// grid (rows, parts / 4)
template <int TYPE>
__global__ __launch_bounds__(kBeamWaves * 64) void k_beam_rows(BeamArgs a, BeamParts p, int parts) {
  using L = Logit<TYPE>;
  constexpr int VE = 16 / L::size, NV = kBeamVals / VE;
  const int r = blockIdx.x, lane = threadIdx.x & 63;
  const int part = blockIdx.y * kBeamWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (part >= parts) return;
  if (a.ended && a.ended[r]) return;  // its logits do not matter
  const int V = a.vocab;
  const uint8_t* row = row_at<TYPE>(a, r);
  // 16 bytes at a time, counted from the row's first token wherever that lies: equal rows have equal
  // sums, and ties between beams are ties.  What is not the row's alone is read by elements.
  float x[kBeamVals];
  uint4 raw[NV];
  auto load = [&](int v) {
    return __builtin_bit_cast(uint4, *(const Raw*)(row + (size_t)((part * NV + v) * 64 + lane) * 16));
  };
  if ((part + 1) * kBeamPart <= V) {
#pragma unroll
    for (int v = 0; v < NV; ++v) raw[v] = load(v);
#pragma unroll
    for (int v = 0; v < NV; ++v) L::spread(raw[v], x + v * VE);
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      raw[v] = uint4{0, 0, 0, 0};
      if (token_of<TYPE>(part, lane, v * VE) + VE <= V) raw[v] = load(v);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int t = token_of<TYPE>(part, lane, v * VE);
      L::spread(raw[v], x + v * VE);
      if (t + VE > V) {
#pragma unroll
        for (int e = 0; e < VE; ++e) x[v * VE + e] = t + e < V ? L::at(row, t + e) : -INFINITY;
      }
    }
  }
  float top = x[0];
#pragma unroll
  for (int i = 1; i < kBeamVals; ++i) top = fmaxf(top, x[i]);
  if (top != top) top = -INFINITY;  // nothing but NaN: the sum says so
  const float m = wave_max(top), base = m == -INFINITY ? 0.f : m;
  double S = 0;
#pragma unroll
  for (int i = 0; i < kBeamVals; i += 8) {
    float s = 0.f;  // NaN and +inf end as NaN
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = x[i + e] - base;
      s += __builtin_amdgcn_exp2f(fmaf(d, kLog2eLo, d * kLog2eHi));
    }
    S += s;
  }
  S = sum64(S);
  const size_t at = (size_t)r * parts + part;
  store_top<TYPE>(p.lanes, at * 64 + lane, top);
  if (lane == 0) {
    p.sums[at] = S;
    p.tops[at] = m;
  }
}

struct Candidate {
  double v;
  int at;  // beam * vocab + token
};

// Order of values as unsigned numbers, larger first; never NaN.
__device__ __forceinline__ u64 value_key(double v) {
  const u64 b = (u64)__double_as_longlong(v + 0.0);
  return b >> 63 ? ~b : b | (1ull << 63);
}

// A sum of e^(x - m) as one of e^(x - to); NaN stays, and an empty one is 0.
__device__ __forceinline__ double weighed(double S, float m, float to) {
  return m == to ? S : m == -INFINITY ? (S != S ? S : 0.0) : S * exp((double)m - (double)to);
}

struct PickShared {
  double m[TSS_BEAMS_MAX], c[TSS_BEAMS_MAX];  // of the beams: NaN c, no candidates
  int state[TSS_BEAMS_MAX];                   // 0: lost, 1: alive, 2: ended
  int beam[TSS_BEAMS_MAX];                    // those alive
  double v[kPickList];
  int at[kPickList];
  int holder[kPickHolders];
  int part[kPickList];
  float top[kPickWaves];
  unsigned cut[kPickWaves], have[kPickWaves];
  float near[kPickThreads], far;
  int n_near;
  int n, holders, parts;
  int bins[256], bin, above;
};

template <int TYPE>
__global__ __launch_bounds__(kPickThreads) void k_beam_pick(BeamArgs a, BeamParts p, int parts) {
  using L = Logit<TYPE>;
  __shared__ PickShared s;
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, B = a.n_beams, V = a.vocab;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = g * B;
  if (tid == 0) s.n = s.holders = s.parts = 0;
  // the rows' sums, a wave each
  for (int b = wave; b < B; b += kPickWaves) {
    const size_t at = (size_t)(row0 + b) * parts;
    const float score = a.scores[row0 + b];
    const bool over = a.ended && a.ended[row0 + b];
    float m = -INFINITY;
    double S = 0;
    if (!over) {
      // a lane's parts one after the other, then the lanes
      float lm = -INFINITY;
      double lS = 0;
#pragma unroll 2
      for (int i = lane; i < parts; i += 64) {
        const float t = p.tops[at + i];
        const double q = p.sums[at + i];
        const float to = fmaxf(lm, t);
        lS = weighed(lS, lm, to) + weighed(q, t, to);
        lm = to;
      }
      m = wave_max(lm);
      S = sum64(weighed(lS, lm, m));
    }
    const bool alive = fabsf(score) < INFINITY && (over || (fabsf(m) < INFINITY && S > 0));
    if (lane == 0) {
      s.m[b] = over ? 0.0 : (double)m;
      s.c[b] = over ? (double)score : (double)score - log(S);
      s.state[b] = !alive ? 0 : over ? 2 : 1;
    }
  }
  __syncthreads();
  auto value = [&](int b, float x) { return (double)x - s.m[b] + s.c[b]; };
  auto list = [&](double v, int at) {
    const int i = atomicAdd(&s.n, 1);
    if (i < kPickList) {
      s.v[i] = v;
      s.at[i] = at;
    }
  };
  auto hold = [&](int id) {
    const int i = atomicAdd(&s.holders, 1);
    if (i < kPickHolders) s.holder[i] = id;
  };
  // a value that the n-th best of the threads' own reaches, so that at least n candidates do
  // (the lowest finite one, where fewer threads have a candidate)
  auto cut_of = [&](double mine) {
    // a little above the best of all
    const float wave_top = wave_max((float)mine);
    const unsigned have = __popcll(__ballot(mine > -INFINITY));
    if (lane == 0) {
      s.top[wave] = wave_top;
      s.have[wave] = have;
    }
    if (tid == 0) s.n_near = 0;
    __syncthreads();
    float top = s.top[0];
    unsigned all = s.have[0];
#pragma unroll
    for (int w = 1; w < kPickWaves; ++w) {
      top = fmaxf(top, s.top[w]);
      all += s.have[w];
    }
    const double best = nextafterf(top, INFINITY);
    // a first cut, as a distance behind the best in fp32 (its 16 upper bits): the need-th of a
    // wave's threads, which has its share of those with candidates
    const unsigned key = mine > -INFINITY ? __float_as_uint((float)(best - mine)) >> 16 : 0xffffu;
    const unsigned need = all >= (unsigned)a.n ? (have * a.n + all - 1) / all : have;
    unsigned cut = 0;  // most keys below it: fewer than need
#pragma unroll
    for (int bit = 15; bit >= 0; --bit) {
      const unsigned c = cut | (1u << bit);
      cut = (unsigned)__popcll(__ballot(key < c)) < need ? c : cut;
    }
    if (lane == 0) s.cut[wave] = need ? cut : 0;
    __syncthreads();
    cut = 0;
#pragma unroll
    for (int w = 0; w < kPickWaves; ++w) cut = max(cut, s.cut[w]);
    // of the threads that reach it (few more than n, for the waves differ), the n-th best is the
    // cut; a distance in fp32 is off by half a step
    double least = -INFINITY;
    if (all >= (unsigned)a.n) {
      if (key <= cut) s.near[atomicAdd(&s.n_near, 1)] = (float)(best - mine);
      __syncthreads();
      const int c = s.n_near;
      for (int i = tid >> 2; i < (c + 15) / 16 * 16; i += kPickThreads / 4) {
        const float d = s.near[min(i, c - 1)];
        int place = 0;
        for (int j = tid & 3; j < c; j += 4) place += s.near[j] < d || (s.near[j] == d && j < i);
        place += __shfl_xor(place, 1);
        place += __shfl_xor(place, 2);
        if (i < c && place == a.n - 1) s.far = d;
      }
      __syncthreads();
      least = s.far < INFINITY ? best - (double)s.far * (1 + 1e-7) : -INFINITY;
    }
    return least == -INFINITY ? kNoCut : least;
  };
  // f(i) for this thread's share of 0 .. count - 1: neighbours go to different waves, so that every
  // wave has some of every beam and its cut is about the group's
  auto share = [&](int count, auto f) {
    for (int i = lane * kPickWaves + wave; i < count; i += kPickThreads) f(i);
  };
  // the beams that can win; lost and ended ones have nothing to look through
  const bool wins = lane < B && s.state[min(lane, B - 1)] == 1;
  const u64 winners = __ballot(wins);
  const int alive = __popcll(winners);
  if (alive < B) {
    if (wave == 0 && wins) s.beam[__popcll(winners & ((1ull << lane) - 1))] = lane;
    __syncthreads();
  }
  const bool by_parts = alive * parts >= kPickParts * a.n;
  const int per = by_parts ? parts : parts * 64, count = alive * per;
  auto place = [&](int i, int& b) {  // of part or lane i of these beams
    const int k = i / per;
    b = alive < B ? s.beam[k] : k;
    return i + (b - k) * per;
  };
  auto lane_top = [&](int b, int id) { return value(b, L::at(p.lanes, (size_t)row0 * parts * 64 + id)); };
  auto grain = [&](int b, int id) { return by_parts ? value(b, p.tops[(size_t)row0 * parts + id]) : lane_top(b, id); };
  auto lanes = [&](auto f) {  // f(place, value) for the lanes of the parts found
    share(s.parts * 64, [&](int i) {
      const int part = s.part[i / 64], id = part * 64 + i % 64;
      f(id, lane_top(part / parts, id));
    });
  };
  double lowest = kNoCut;
  bool fits;
  for (int again = 0;; again = 1) {
    double mine = -INFINITY;
    if (again) {
      lanes([&](int, double v) { mine = fmax(mine, v); });
    } else {
      share(count, [&](int i) {
        int b;
        const int id = place(i, b);
        mine = fmax(mine, grain(b, id));
      });
    }
    lowest = fmax(lowest, cut_of(mine));
    if (again) {
      if (tid == 0) s.holders = 0;
    } else {
      if (tid < B && s.state[tid] == 2) list(s.c[tid], tid * V + a.end_token);
      share(count, [&](int i) {
        int b;
        const int id = place(i, b);
        if (!((count <= kPickThreads ? mine : grain(b, id)) >= lowest)) return;
        if (by_parts) {
          const int k = atomicAdd(&s.parts, 1);
          if (k < kPickList) s.part[k] = id;
        } else {
          hold(id);
        }
      });
    }
    __syncthreads();
    fits = s.parts <= kPickList;
    if (!by_parts || !fits) break;
    lanes([&](int id, double v) {
      if (v >= lowest) hold(id);
    });
    __syncthreads();
    // where many lanes reach the parts' cut (or there was none), the best candidates are in few of the
    // parts (scores far apart, masked logits): it is sought again, among their lanes
    if (again || s.holders <= (lowest == kNoCut ? kPickList / kBeamVals : kPickMany)) break;
  }
  fits = fits && s.holders <= kPickHolders;
  if (fits) {
    for (int i = tid; i < s.holders * kBeamVals; i += kPickThreads) {
      const int id = s.holder[i / kBeamVals], b = id / (parts * 64);
      const uint8_t* row = row_at<TYPE>(a, row0 + b);
      const int t = token_of<TYPE>(id / 64 % parts, id % 64, i % kBeamVals);
      if (t >= V) continue;
      const double v = value(b, L::at(row, t));
      if (v >= lowest) list(v, b * V + t);
    }
    __syncthreads();
    fits = s.n <= kPickList;
  }
  auto each = [&](auto f) {  // f(value, place) for this thread's share of the group's candidates
    for (int b = 0; b < B; ++b) {
      if (s.state[b] == 1) {
        const uint8_t* row = row_at<TYPE>(a, row0 + b);
        for (int t = tid; t < V; t += kPickThreads) {
          const double v = value(b, L::at(row, t));
          if (v >= lowest) f(v, b * V + t);
        }
      } else if (s.state[b] == 2 && tid == 0) {
        f(s.c[b], b * V + a.end_token);
      }
    }
  };
  if (!fits) {
    // the least prefix of (value, place) that at least n candidates reach, 8 bits longer each
    // time, until few enough do
    __syncthreads();
    u64 prefix = 0;
    unsigned low = 0;  // place's bits, inverted: the lower place is the larger
    int above = 0;
    int shift = 88;
    for (; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kPickThreads) s.bins[i] = 0;
      __syncthreads();
      each([&](double v, int at) {
        const u64 k = value_key(v);
        const unsigned q = ~(unsigned)at;
        if (shift >= 32) {
          const int sh = shift - 32;
          if (sh == 56 || k >> (sh + 8) == prefix >> (sh + 8)) atomicAdd(&s.bins[(k >> sh) & 255], 1);
        } else if (k == prefix && (shift == 24 || q >> (shift + 8) == low >> (shift + 8))) {
          atomicAdd(&s.bins[(q >> shift) & 255], 1);
        }
      });
      __syncthreads();
      if (tid == 0) {
        int b = 255, over = above;
        while (b > 0 && over + s.bins[b] < a.n) over += s.bins[b--];
        s.bin = b;
        s.above = over;
      }
      __syncthreads();
      above = s.above;
      if (shift >= 32)
        prefix |= (u64)s.bin << (shift - 32);
      else
        low |= (unsigned)s.bin << shift;
      const int reach = above + s.bins[s.bin];
      __syncthreads();
      if (reach <= kPickList) break;
    }
    if (tid == 0) s.n = 0;
    __syncthreads();
    each([&](double v, int at) {
      const u64 k = value_key(v);
      if (k > prefix || (k == prefix && ~(unsigned)at >= low)) list(v, at);
    });
    __syncthreads();
  }
  int n = min(s.n, kPickList);
  if (n < a.n) {
    // fewer candidates than are asked for: behind them pairs of -inf by their place, which
    // are among the first a.n pairs
    __syncthreads();
    if (tid < a.n) {
      const int b = tid / V, t = tid % V;
      bool none = s.state[b] != 1;
      if (s.state[b] == 2) none = t != a.end_token;
      if (s.state[b] == 1) none = !(value(b, L::at(row_at<TYPE>(a, row0 + b), t)) >= lowest);
      if (none) list(-INFINITY, tid);
    }
    __syncthreads();
    n = min(s.n, kPickList);
  }
  // four lanes count what precedes a candidate
  for (int i = tid >> 2; i < (n + 15) / 16 * 16; i += kPickThreads / 4) {
    const double v = s.v[min(i, n - 1)];
    const int at = s.at[min(i, n - 1)];
    int place = 0;
    for (int j = tid & 3; j < n; j += 4) place += s.v[j] > v || (s.v[j] == v && s.at[j] < at);
    place += __shfl_xor(place, 1);
    place += __shfl_xor(place, 2);
    if (i < n && place < a.n && (tid & 3) == 0) {
      const size_t o = (size_t)g * a.n + place;
      a.score[o] = (float)v;
      a.parent[o] = at / V;
      a.token[o] = at % V;
    }
  }
}

size_t align16(size_t n) { return (n + 15) & ~(size_t)15; }

int parts_of(int vocab) { return (vocab + kBeamPart - 1) / kBeamPart; }

}  // namespace

bool beams_fit(int n_groups, int n_beams, int vocab) {
  return vocab <= kLogprobVocab && (int64_t)n_groups * n_beams * ((parts_of(vocab) + 3) / 4) <= (1 << 22);
}

size_t beams_bytes(int n_groups, int n_beams, int vocab, int) {
  const size_t c = (size_t)n_groups * n_beams * parts_of(vocab);
  return align16(c * 8) + align16(c * 4) + c * 64 * 4;
}

template <int TYPE>
static hipError_t launch_typed(const BeamArgs& a, uint8_t* ws, hipStream_t s) {
  const int parts = parts_of(a.vocab), rows = a.n_groups * a.n_beams;
  const size_t c = (size_t)rows * parts;
  BeamParts p{(double*)ws, (float*)(ws + align16(c * 8)), ws + align16(c * 8) + align16(c * 4)};
  const int y = (parts + kBeamWaves - 1) / kBeamWaves;
  TSS_LAUNCH(k_beam_rows<TYPE>, dim3(rows, y), dim3(kBeamWaves * 64), 0, s, a, p, parts);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  TSS_LAUNCH(k_beam_pick<TYPE>, dim3(a.n_groups), dim3(kPickThreads), 0, s, a, p, parts);
  return hipGetLastError();
}

hipError_t launch_beams(const BeamArgs& a, void* ws, hipStream_t s) {
  if (a.n_groups < 1 || a.n_beams < 1 || a.n_beams > TSS_BEAMS_MAX || a.vocab < 1 || a.n < 1 ||
      a.n > TSS_BEAMS_MAX_N || !beams_fit(a.n_groups, a.n_beams, a.vocab))
    return hipErrorInvalidValue;
  uint8_t* w = (uint8_t*)ws;
  if (a.type == TSS_T_F32) return launch_typed<TSS_T_F32>(a, w, s);
  if (a.type == TSS_T_F16) return launch_typed<TSS_T_F16>(a, w, s);
  return launch_typed<TSS_T_BF16>(a, w, s);
}

}  // namespace tss
