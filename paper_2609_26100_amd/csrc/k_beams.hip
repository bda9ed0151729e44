// The n best continuations of each group of beams (gfx950).
//
// A candidate (beam b, token t) is worth scores[b] + x[b][t] - ln sum e^x[b].  One
// launch takes each row's logarithm of the sum, a second picks the n best of a group
// one after the other.
#include "../../include/tss.h"
#include "tss_internal.h"

namespace tss {

namespace {

constexpr int kBeamThreads = 1024;

template <int TYPE>
__device__ __forceinline__ float logit(const void* p, size_t i) {
  if constexpr (TYPE == TSS_T_F32) return ((const float*)p)[i];
  if constexpr (TYPE == TSS_T_F16) return (float)((const _Float16*)p)[i];
  return __uint_as_float((unsigned)((const uint16_t*)p)[i] << 16);
}

// A beam's candidates are worth (x - m) + c: m its largest logit, c its score less the
// logarithm (m is taken off first, for far from zero its sum with c would lose c); c is
// NaN for a beam without candidates.
struct Base {
  double m, c;
};

template <int TYPE>
__global__ __launch_bounds__(kBeamThreads) void k_beam_rows(BeamArgs a, Base* base) {
  __shared__ float s_m[kBeamThreads];
  __shared__ double s_s[kBeamThreads];
  const int r = blockIdx.x, tid = threadIdx.x;
  const size_t es = TYPE == TSS_T_F32 ? 4 : 2;
  const uint8_t* row = (const uint8_t*)a.x + (size_t)r * a.stride * es;
  float m = -INFINITY;
  bool bad = false;
  for (int t = tid; t < a.vocab; t += kBeamThreads) {
    const float x = logit<TYPE>(row, t);
    bad |= !(x < INFINITY);
    m = fmaxf(m, x);
  }
  s_m[tid] = bad ? INFINITY : m;
  __syncthreads();
  for (int w = kBeamThreads / 2; w > 0; w >>= 1) {
    if (tid < w) s_m[tid] = fmaxf(s_m[tid], s_m[tid + w]);
    __syncthreads();
  }
  m = s_m[0];
  double sum = 0;
  if (fabsf(m) < INFINITY)
    for (int t = tid; t < a.vocab; t += kBeamThreads) sum += expf(logit<TYPE>(row, t) - m);
  s_s[tid] = sum;
  __syncthreads();
  for (int w = kBeamThreads / 2; w > 0; w >>= 1) {
    if (tid < w) s_s[tid] += s_s[tid + w];
    __syncthreads();
  }
  if (tid == 0) {
    const float score = a.scores[r];
    const bool over = a.ended && a.ended[r];
    Base b{over ? 0.0 : (double)m, over ? (double)score : (double)score - log(s_s[0])};
    if (!(fabsf(score) < INFINITY) || (!over && !(fabsf(m) < INFINITY))) b.c = __builtin_nan("");
    base[r] = b;
  }
}

struct Best {
  double v;
  int64_t at;  // beam * vocab + token
  __device__ bool before(const Best& o) const { return v > o.v || (v == o.v && at < o.at); }
};

template <int TYPE>
__global__ __launch_bounds__(kBeamThreads) void k_beam_pick(BeamArgs a, const Base* base) {
  __shared__ Best s_b[kBeamThreads];
  const int g = blockIdx.x, tid = threadIdx.x;
  const size_t es = TYPE == TSS_T_F32 ? 4 : 2;
  Best last{INFINITY, -1};
  for (int i = 0; i < a.n; ++i) {
    Best best{-INFINITY, INT64_MAX};
    for (int b = 0; b < a.n_beams; ++b) {
      const int r = g * a.n_beams + b;
      const Base add = base[r];
      const bool over = a.ended && a.ended[r];
      for (int t = tid; t < a.vocab; t += kBeamThreads) {
        double v = over ? (t == a.end_token ? add.c : -INFINITY)
                        : (double)logit<TYPE>((const uint8_t*)a.x + (size_t)r * a.stride * es, t) - add.m + add.c;
        if (v != v) v = -INFINITY;
        const Best c{v, (int64_t)b * a.vocab + t};
        if (last.before(c) && c.before(best)) best = c;
      }
    }
    s_b[tid] = best;
    __syncthreads();
    for (int w = kBeamThreads / 2; w > 0; w >>= 1) {
      if (tid < w && s_b[tid + w].before(s_b[tid])) s_b[tid] = s_b[tid + w];
      __syncthreads();
    }
    last = s_b[0];
    __syncthreads();
    if (tid == 0) {
      const size_t o = (size_t)g * a.n + i;
      a.score[o] = (float)last.v;
      a.parent[o] = (int)(last.at / a.vocab);
      a.token[o] = (int)(last.at % a.vocab);
    }
  }
}

}  // namespace

bool beams_fit(int n_groups, int n_beams, int vocab) {
  return vocab <= kLogprobVocab && (int64_t)n_groups * n_beams <= (1 << 22);
}

size_t beams_bytes(int n_groups, int n_beams, int, int) { return (size_t)n_groups * n_beams * sizeof(Base); }

template <int TYPE>
static hipError_t launch_typed(const BeamArgs& a, Base* ws, hipStream_t s) {
  TSS_LAUNCH(k_beam_rows<TYPE>, dim3(a.n_groups * a.n_beams), dim3(kBeamThreads), 0, s, a, ws);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  TSS_LAUNCH(k_beam_pick<TYPE>, dim3(a.n_groups), dim3(kBeamThreads), 0, s, a, (const Base*)ws);
  return hipGetLastError();
}

hipError_t launch_beams(const BeamArgs& a, void* ws, hipStream_t s) {
  if (a.n_groups < 1 || a.n_beams < 1 || a.vocab < 1) return hipErrorInvalidValue;
  if (a.type == TSS_T_F32) return launch_typed<TSS_T_F32>(a, (Base*)ws, s);
  if (a.type == TSS_T_F16) return launch_typed<TSS_T_F16>(a, (Base*)ws, s);
  return launch_typed<TSS_T_BF16>(a, (Base*)ws, s);
}

}  // namespace tss
