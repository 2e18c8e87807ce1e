// Scores of logits rows: log probabilities of given tokens, the entropy, the
// normaliser and the most likely tokens.
//
// One pass over a row: every thread keeps the running maximum m of its values,
// the sum S of exp(x - m) and T of exp(x - m) (x - m), rescaled when m grows;
// joined over the workgroup, lse = m + log S and the entropy is log S - T / S.
// The k largest values come out of the same pass.  The first tile of the row
// gives a lower bound of the k-th largest value (the k-th largest of 256
// groups' maxima: about as many values as k lie above it in the tile); every
// value from the bound on joins a list in LDS, which is sorted at the end by
// counting for each entry those before it.  A row whose later tiles hold more
// than the list does (values in rising order, say) is read once more in steps
// that cut the list back to its k best.
#include "batch.h"

namespace llmcad {

namespace {

constexpr int kScoreThreads = 1024;
constexpr int kScoreWaves = kScoreThreads / kWave;
constexpr int kPer = 16;                           // values per thread and tile
constexpr int kTile = kPer * kScoreThreads;
constexpr int kList = 2048;
constexpr float kLowest = -3.402823466e38f;        // (finite: x - m stays a number for rows of -inf)
constexpr float kLog2e = 1.4426950408889634f;

struct ScoreLds {
  float m[kScoreWaves], s[kScoreWaves], t[kScoreWaves];
  float group[256];
  float bound;
  int count;
  uint64_t list[kList];  // ordered value bits << 32 | ~token: larger is better, ties to the lower token
  uint64_t keep[LLMCAD_TOP_MAX];
};

// Bits of a float in the floats' order (no NaN).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);  // (-0 ties with 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

// Values [i0, i0 + N) of the row (i0 may be negative, i0 + N past V: -inf
// there); 16-byte loads where all of them are the row's (row + i0 is then
// 16-byte aligned).
template <bool BF16>
__device__ __forceinline__ void load16(const void* row, long i0, int V, float* x) {
  constexpr int N = BF16 ? 8 : 4;
  if (i0 >= 0 && i0 + N <= V) {
    if (BF16) {
      const bf16x8 v = ldg((const bf16x8*)((const bf16*)row + i0));
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = bf2f(v[e]);
    } else {
      const f32x4 v = ldg((const f32x4*)((const float*)row + i0));
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = v[e];
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const long i = i0 + e;
    x[e] = -INFINITY;
    if (i >= 0 && i < V) x[e] = BF16 ? bf2f(ldg((const bf16*)row + i)) : ldg((const float*)row + i);
  }
}

template <bool BF16>
__device__ __forceinline__ void load_tile(const void* row, long base, int V, float (&x)[kPer]) {
  constexpr int N = BF16 ? 8 : 4;
#pragma unroll
  for (int v = 0; v < kPer / N; ++v)
    load16<BF16>(row, base + (long)v * N * kScoreThreads + N * threadIdx.x, V, x + v * N);
}
// Token of value e of this thread's tile at base.
template <bool BF16>
__device__ __forceinline__ long tile_token(long base, int e) {
  constexpr int N = BF16 ? 8 : 4;
  return base + (long)(e / N) * N * kScoreThreads + N * threadIdx.x + e % N;
}

template <bool BF16>
__device__ __forceinline__ float value_at(const void* row, int i) {
  return BF16 ? bf2f(ldg((const bf16*)row + i)) : ldg((const float*)row + i);
}

// The list's k best, sorted, in L.keep (0: no entry).  All threads call it.
__device__ __forceinline__ void keep_best(ScoreLds& L, int count, int k) {
  if (threadIdx.x < k) L.keep[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += kScoreThreads) {
    const uint64_t mine = L.list[i];
    int before = 0;
    for (int j = 0; j < count; ++j) before += L.list[j] > mine ? 1 : 0;
    if (before < k) L.keep[before] = mine;
  }
  __syncthreads();
}

// The k best of a row whose list overflowed.
template <bool BF16>
__device__ __attribute__((noinline)) void best_in_steps(const void* row, int V, int k, ScoreLds& L) {
  uint64_t least = 0;  // the k-th best so far: later entries must be larger
  __syncthreads();
  if (threadIdx.x == 0) L.count = 0;
  for (long i0 = 0; i0 < V; i0 += kScoreThreads) {
    __syncthreads();
    const long i = i0 + threadIdx.x;
    if (i < V) {
      const float x = value_at<BF16>(row, (int)i);
      const uint64_t key = (uint64_t)ordered(x) << 32 | (uint32_t)~(uint32_t)i;
      if (x > -INFINITY && key > least) L.list[atomicAdd(&L.count, 1)] = key;
    }
    __syncthreads();
    const int count = L.count;
    if (count > kList - kScoreThreads) {
      keep_best(L, count, k);
      if (threadIdx.x < k) L.list[threadIdx.x] = L.keep[threadIdx.x];
      if (threadIdx.x == 0) L.count = k;
      least = L.keep[k - 1];
    }
  }
  __syncthreads();
  keep_best(L, L.count, k);
}

template <bool BF16>
__global__ __launch_bounds__(kScoreThreads) void scores_kernel(ScoresArgs a) {
  __shared__ ScoreLds L;
  const int r = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, V = a.V, k = a.k;
  constexpr int ESIZE = BF16 ? 2 : 4;
  const char* row = (const char*)a.logits + (size_t)r * a.stride * ESIZE;
  // tiles start on the 16-byte boundary at or before the row
  const long lead = (long)(((uintptr_t)row & 15) / ESIZE);
  if (tid == 0) {
    L.count = 0;
    L.bound = -INFINITY;
  }
  float m = kLowest, S = 0.0f, T = 0.0f, bound = -INFINITY;
  float x[kPer], nx[kPer];
  load_tile<BF16>(row, -lead, V, nx);
  for (long base = -lead; base < V; base += kTile) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) x[e] = nx[e];
    if (base + kTile < V) load_tile<BF16>(row, base + kTile, V, nx);
    float top = x[0];
#pragma unroll
    for (int e = 1; e < kPer; ++e) top = fmaxf(top, x[e]);
    const float grown = fmaxf(m, top);
    const float step = fmaxf(m - grown, -1e4f);  // (0 where the maximum stays)
    const float alpha = __builtin_amdgcn_exp2f(step * kLog2e);
    T = alpha * (T + S * step);
    S = alpha * S;
    m = grown;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const float d = x[e] - m;  // (NaN for NaN and +inf: S tells)
      const float p = __builtin_amdgcn_exp2f(d * kLog2e);
      S += p;
      T += p * fmaxf(d, -1e4f);  // (0 (-inf) is no number)
    }
    if (k > 0) {
      if (base <= 0) {  // the first tile: the bound
        float g = top;
        g = fmaxf(g, __shfl_xor(g, 1, kWave));
        g = fmaxf(g, __shfl_xor(g, 2, kWave));
        if ((tid & 3) == 0) L.group[tid >> 2] = g;
        __syncthreads();
        if (tid < 256) {
          const float mine = L.group[tid];
          int before = 0;
          for (int j = 0; j < 256; ++j) {
            const float o = L.group[j];
            before += o > mine || (o == mine && j < tid) ? 1 : 0;
          }
          if (before == k - 1) L.bound = mine;
        }
        __syncthreads();
        bound = L.bound;
      }
      if (top >= bound && top > -INFINITY) {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          if (x[e] >= bound && x[e] > -INFINITY) {
            const int at = atomicAdd(&L.count, 1);
            if (at < kList) L.list[at] = (uint64_t)ordered(x[e]) << 32 | (uint32_t)~(uint32_t)tile_token<BF16>(base, e);
          }
      }
    }
  }
  // (m, S, T) over the workgroup: lanes, then waves in order
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const float om = __shfl_xor(m, off, kWave), os = __shfl_xor(S, off, kWave), ot = __shfl_xor(T, off, kWave);
    const float mm = fmaxf(m, om), da = fmaxf(m - mm, -1e4f), db = fmaxf(om - mm, -1e4f);
    const float ea = __builtin_amdgcn_exp2f(da * kLog2e), eb = __builtin_amdgcn_exp2f(db * kLog2e);
    T = ea * (T + S * da) + eb * (ot + os * db);
    S = ea * S + eb * os;
    m = mm;
  }
  if ((tid & 63) == 0) {
    L.m[wave] = m;
    L.s[wave] = S;
    L.t[wave] = T;
  }
  __syncthreads();
  m = kLowest;
  for (int w = 0; w < kScoreWaves; ++w) m = fmaxf(m, L.m[w]);
  S = T = 0.0f;
  for (int w = 0; w < kScoreWaves; ++w) {
    const float d = fmaxf(L.m[w] - m, -1e4f), e = __builtin_amdgcn_exp2f(d * kLog2e);
    T += e * (L.t[w] + L.s[w] * d);
    S += e * L.s[w];
  }
  const bool none = S == 0.0f, bad = S != S;
  const float logS = none ? 0.0f : logf(S);
  const float lse = bad ? S : none ? -INFINITY : m + logS;
  if (tid == 0) {
    stg(a.lse + r, lse);
    stg(a.entropy + r, bad ? S : none ? 0.0f : logS - T / S);
  }
  // the given tokens under this row
  auto score = [&](int q) {
    const int t = ldg(a.tokens + q);
    float v = 0.0f;
    if (t >= V) v = NAN;
    else if (t >= 0) v = bad ? S : none ? -INFINITY : (value_at<BF16>(row, t) - m) - logS;
    stg(a.logprob + q, v);
  };
  if (a.row_of == nullptr) {
    if (tid == 0 && r < a.m) score(r);
  } else {
    for (int q = tid; q < a.m; q += kScoreThreads) {
      const int of = ldg(a.row_of + q);
      if (of == r) score(q);
      else if (r == 0 && (of < 0 || of >= a.n)) stg(a.logprob + q, (float)NAN);
    }
  }
  if (k == 0) return;
  const int count = L.count;  // (the last addition lies before the barrier above)
  if (bad) {
    if (tid < k) L.keep[tid] = 0;
  } else if (count <= kList) {
    keep_best(L, count, k);
  } else {
    best_in_steps<BF16>(row, V, k, L);
  }
  if (tid < k) {
    const uint64_t e = L.keep[tid];
    stg(a.top_token + (size_t)r * k + tid, e ? (int)~(uint32_t)e : -1);
    stg(a.top_logprob + (size_t)r * k + tid, bad ? S : e ? (unordered((uint32_t)(e >> 32)) - m) - logS : -INFINITY);
  }
}

}  // namespace

hipError_t launch_token_scores(const ScoresArgs& a, hipStream_t st) {
  if (a.bf16_in)
    scores_kernel<true><<<dim3(a.n), dim3(kScoreThreads), 0, st>>>(a);
  else
    scores_kernel<false><<<dim3(a.n), dim3(kScoreThreads), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace llmcad
