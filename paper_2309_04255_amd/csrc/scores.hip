// Scores of logits rows: log probabilities of given tokens, the entropy, the
// normaliser and the most likely tokens.
//
// One pass over a row, the next tile's loads in flight while one is computed:
// every thread keeps the running maximum m of its values, the sum S of exp(x - m)
// and T of exp(x - m) (x - m), rescaled when m grows; joined over the workgroup,
// lse = m + log S and the entropy is log S - T / S.  The k largest values come out
// of the same pass.  The first tile gives a lower bound of the k-th largest value
// (the k-th largest of 256 groups' maxima: about as many values as k lie above it
// in the tile); every value from the bound on joins a list in LDS.  After 2, 4, 8
// .. tiles the list's k-th best becomes the bound, so that a row adds about
// k log(tiles) entries; at the end the list is sorted by counting for each entry
// those before it.  A row whose later tiles hold more than the list does (values
// in rising order, say) is read once more in steps that cut the list back to its
// k best.
#include "batch.h"

namespace llmcad {

namespace {

constexpr int kPieces = 4;  // 16-byte pieces of a row per thread and tile
constexpr int kList = 2048;
constexpr int kGroups = 256;
constexpr float kLowest = -3.402823466e38f;        // (finite: x - m stays a number for rows of -inf)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct ScoreLds {
  float m[16], s[16], t[16];  // by wave
  __align__(16) float group[kGroups];
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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A thread's part of the tile at base: pieces of 16 bytes, kPieces of them a
// workgroup's width apart, as they lie in memory.  (row + base is 16-byte aligned;
// what lies outside the row, before its first or behind its last value, reads as
// -inf and is not touched.)
template <bool BF16, int THREADS>
struct Tile {
  static constexpr int N = BF16 ? 8 : 4;             // values per piece
  static constexpr int PER = N * kPieces;            // values per thread
  static constexpr int SIZE = PER * THREADS;
  u32x4 raw[kPieces];

  __device__ static __forceinline__ long at(long base, int piece) { return base + (long)N * (piece * THREADS + (int)threadIdx.x); }
  __device__ __forceinline__ void load(const char* row, long base, int V) {
    constexpr int ES = 16 / N;
    if (base >= 0 && base + SIZE <= V) {
#pragma unroll
      for (int v = 0; v < kPieces; ++v) raw[v] = ldg((const u32x4*)(row + at(base, v) * ES));
      return;
    }
#pragma unroll
    for (int v = 0; v < kPieces; ++v) {
      const long i0 = at(base, v);
      const uint32_t none = BF16 ? 0xff80ff80u : 0xff800000u;
      u32x4 x = {none, none, none, none};
      if (i0 >= 0 && i0 + N <= V) {
        x = ldg((const u32x4*)(row + i0 * ES));
      } else if (i0 < V) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const long i = i0 + e;
          if (i < 0 || i >= V) continue;
          if (BF16) {
            const uint32_t bits = ldg((const uint16_t*)row + i);
            x[e / 2] = e & 1 ? (x[e / 2] & 0xffffu) | bits << 16 : (x[e / 2] & 0xffff0000u) | bits;
          } else {
            x[e & 3] = ldg((const uint32_t*)row + i);
          }
        }
      }
      raw[v] = x;
    }
  }
  __device__ __forceinline__ float value(int e) const {  // value e of the thread's PER
    const uint32_t w = raw[e / N][BF16 ? (e % N) / 2 : e % N];
    return __uint_as_float(!BF16 ? w : e & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ static __forceinline__ long token(long base, int e) { return at(base, e / N) + e % N; }
};

template <bool BF16>
__device__ __forceinline__ float value_at(const void* row, int i) {
  return BF16 ? bf2f(ldg((const bf16*)row + i)) : ldg((const float*)row + i);
}

// The list's k best, sorted, in L.keep (0: no entry).  All threads call it;
// groups of neighbouring lanes count for one entry together.
template <int THREADS>
__device__ __forceinline__ void keep_best(ScoreLds& L, int count, int k) {
  if (threadIdx.x < k) L.keep[threadIdx.x] = 0;
  __syncthreads();
  int share = kWave;  // lanes per entry
  while (share > 1 && count * share > THREADS) share >>= 1;
  const int part = threadIdx.x & (share - 1);
  for (int i0 = 0; i0 < count; i0 += THREADS / share) {
    const int i = i0 + threadIdx.x / share;
    const uint64_t mine = i < count ? L.list[i] : 0;
    int before = 0;
    if (i < count)
      for (int j = part; j < count; j += share) before += L.list[j] > mine ? 1 : 0;
    for (int off = share >> 1; off >= 1; off >>= 1) before += __shfl_xor(before, off, kWave);
    if (i < count && part == 0 && before < k) L.keep[before] = mine;
  }
  __syncthreads();
}

// The list's k-th best value (L.bound), if it has k entries.  All threads call it.
template <int THREADS>
__device__ __forceinline__ void raise_bound(ScoreLds& L, int k) {
  __syncthreads();
  const int count = L.count;
  __syncthreads();  // (nobody adds before all have read the count)
  if (count >= k && count <= kList) {
    int share = kWave;
    while (share > 1 && count * share > THREADS) share >>= 1;
    const int part = threadIdx.x & (share - 1);
    for (int i0 = 0; i0 < count; i0 += THREADS / share) {
      const int i = i0 + threadIdx.x / share;
      const uint64_t mine = i < count ? L.list[i] : 0;
      int before = 0;
      if (i < count)
        for (int j = part; j < count; j += share) before += L.list[j] > mine ? 1 : 0;
      for (int off = share >> 1; off >= 1; off >>= 1) before += __shfl_xor(before, off, kWave);
      if (i < count && part == 0 && before == k - 1) L.bound = unordered((uint32_t)(mine >> 32));
    }
  }
  __syncthreads();
}

// The k best of a row whose list overflowed.
template <bool BF16, int THREADS>
__device__ __attribute__((noinline)) void best_in_steps(const void* row, int V, int k, ScoreLds& L) {
  uint64_t least = 0;  // the k-th best so far: later entries must be larger
  __syncthreads();
  if (threadIdx.x == 0) L.count = 0;
  for (long i0 = 0; i0 < V; i0 += THREADS) {
    __syncthreads();
    const long i = i0 + threadIdx.x;
    if (i < V) {
      const float x = value_at<BF16>(row, (int)i);
      const uint64_t key = (uint64_t)ordered(x) << 32 | (uint32_t)~(uint32_t)i;
      if (x > -INFINITY && key > least) L.list[atomicAdd(&L.count, 1)] = key;
    }
    __syncthreads();
    const int count = L.count;
    if (count > kList - THREADS) {
      keep_best<THREADS>(L, count, k);
      if (threadIdx.x < k) L.list[threadIdx.x] = L.keep[threadIdx.x];
      if (threadIdx.x == 0) L.count = k;
      least = L.keep[k - 1];
    }
  }
  __syncthreads();
  keep_best<THREADS>(L, L.count, k);
}

// A maximum m, S = sum of exp(x - m) and T = sum of exp(x - m) (x - m).
struct Sums {
  float m, s, t;
};
// The same over the workgroup: lanes, then waves in order.  unit: log2 of the base
// that the sums are in.  All threads call it.
template <int THREADS>
__device__ __forceinline__ void join(ScoreLds& L, Sums& w, float unit) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const float om = __shfl_xor(w.m, off, kWave), os = __shfl_xor(w.s, off, kWave), ot = __shfl_xor(w.t, off, kWave);
    const float mm = fmaxf(w.m, om), da = fmaxf(w.m - mm, -1e4f), db = fmaxf(om - mm, -1e4f);
    const float ea = __builtin_amdgcn_exp2f(da * unit), eb = __builtin_amdgcn_exp2f(db * unit);
    w.t = ea * (w.t + w.s * da) + eb * (ot + os * db);
    w.s = ea * w.s + eb * os;
    w.m = mm;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) {
    L.m[threadIdx.x >> 6] = w.m;
    L.s[threadIdx.x >> 6] = w.s;
    L.t[threadIdx.x >> 6] = w.t;
  }
  __syncthreads();
  w.m = L.m[0];
  for (int i = 1; i < THREADS / kWave; ++i) w.m = fmaxf(w.m, L.m[i]);
  w.s = w.t = 0.0f;
  for (int i = 0; i < THREADS / kWave; ++i) {
    const float d = fmaxf(L.m[i] - w.m, -1e4f), e = __builtin_amdgcn_exp2f(d * unit);
    w.t += e * (L.t[i] + L.s[i] * d);
    w.s += e * L.s[i];
  }
}

// The sums of a row in natural units, which hold for every finite value.
template <bool BF16, int THREADS>
__device__ __attribute__((noinline)) Sums sums_again(const void* row, int V, ScoreLds& L) {
  Sums w = {kLowest, 0.0f, 0.0f};
  for (int i = threadIdx.x; i < V; i += THREADS) {
    const float x = value_at<BF16>(row, i), grown = fmaxf(w.m, x), step = fmaxf(w.m - grown, -1e4f);
    const float alpha = __builtin_amdgcn_exp2f(step * kLog2e);
    const float d = x - grown, p = __builtin_amdgcn_exp2f(d * kLog2e);  // (NaN for NaN and +inf)
    w.t = alpha * (w.t + w.s * step) + p * fmaxf(d, -1e4f);
    w.s = alpha * w.s + p;
    w.m = grown;
  }
  join<THREADS>(L, w, kLog2e);
  return w;
}

template <bool BF16, int THREADS>
__global__ __launch_bounds__(THREADS) void scores_kernel(ScoresArgs a) {
  typedef Tile<BF16, THREADS> T_;
  __shared__ ScoreLds L;
  const int r = blockIdx.x, tid = threadIdx.x, V = a.V, k = a.k;
  constexpr int ESIZE = BF16 ? 2 : 4;
  const char* row = (const char*)a.logits + (size_t)r * a.stride * ESIZE;
  // tiles start on the 16-byte boundary at or before the row
  const long lead = (long)(((uintptr_t)row & 15) / ESIZE);
  if (tid == 0) {
    L.count = 0;
    L.bound = -INFINITY;
  }
  Sums w = {-1e37f, 0.0f, 0.0f};  // (in the log2 domain: one product less per value)
  float bound = -INFINITY;
  T_ tile, ahead;
  ahead.load(row, -lead, V);
  int done = 0;  // tiles
  for (long base = -lead; base < V; base += T_::SIZE) {
    tile = ahead;
    if (base + T_::SIZE < V) ahead.load(row, base + T_::SIZE, V);
    float tops[kPieces], top = -INFINITY;  // largest values of the pieces, of all
#pragma unroll
    for (int v = 0; v < kPieces; ++v) {
      tops[v] = tile.value(v * T_::N);
#pragma unroll
      for (int e = 1; e < T_::N; ++e) tops[v] = fmaxf(tops[v], tile.value(v * T_::N + e));
      top = fmaxf(top, tops[v]);
    }
    const float grown = fmaxf(w.m, top * kLog2e);
    const float step = fmaxf(w.m - grown, -1e4f);  // (0 where the maximum stays)
    const float alpha = __builtin_amdgcn_exp2f(step);
    w.t = alpha * (w.t + w.s * step);
    w.s = alpha * w.s;
    w.m = grown;
#pragma unroll
    for (int e = 0; e < T_::PER; ++e) {
      const float d = __builtin_fmaf(tile.value(e), kLog2e, -w.m);
      const float p = __builtin_amdgcn_exp2f(d);
      w.s += p;
      w.t += p * fmaxf(d, -1e4f);  // (0 (-inf) is no number)
    }
    if (k > 0) {
      if (done == 0) {  // the first tile: the bound
        constexpr int PER_GROUP = THREADS / kGroups;
        float gm = top;
#pragma unroll
        for (int off = 1; off < PER_GROUP; off <<= 1) gm = fmaxf(gm, __shfl_xor(gm, off, kWave));
        const int group = tid / PER_GROUP, part = tid % PER_GROUP;
        if (part == 0) L.group[group] = gm;
        __syncthreads();
        int before = 0;  // the groups before this one, a share of them per lane
#pragma unroll 4
        for (int j = part * (kGroups / PER_GROUP); j < (part + 1) * (kGroups / PER_GROUP); j += 4) {
          const f32x4 o = *(const f32x4*)&L.group[j];
#pragma unroll
          for (int e = 0; e < 4; ++e) before += o[e] > gm || (o[e] == gm && j + e < group) ? 1 : 0;
        }
#pragma unroll
        for (int off = 1; off < PER_GROUP; off <<= 1) before += __shfl_xor(before, off, kWave);
        if (part == 0 && before == k - 1) L.bound = gm;
        __syncthreads();
        bound = fmaxf(L.bound, kLowest);  // (-inf is no alternative)
      }
#pragma unroll
      for (int v = 0; v < kPieces; ++v) {
        if (!__any(tops[v] >= bound)) continue;
#pragma unroll
        for (int e = v * T_::N; e < (v + 1) * T_::N; ++e) {
          const float x = tile.value(e);
          const uint64_t hits = __ballot(x >= bound);
          if (hits == 0) continue;
          const int lane = tid & 63, first = __ffsll((unsigned long long)hits) - 1;
          int at = 0;
          if (lane == first) at = atomicAdd(&L.count, __popcll(hits));
          at = __builtin_amdgcn_readlane(at, first) + __popcll(hits & ((1ull << lane) - 1));
          if (x >= bound && at < kList) L.list[at] = (uint64_t)ordered(x) << 32 | (uint32_t)~(uint32_t)T_::token(base, e);
        }
      }
      ++done;
      if (done > 1 && (done & (done - 1)) == 0 && base + T_::SIZE < V) {
        raise_bound<THREADS>(L, k);
        bound = fmaxf(L.bound, kLowest);
      }
    }
  }
  join<THREADS>(L, w, 1.0f);
  // A sum of 0 or NaN: a row of nothing but -inf, with a NaN or +inf -- or with
  // values so large that their log2 is no fp32 number.
  const bool plain = w.s > 0.0f;
  if (!plain) w = sums_again<BF16, THREADS>(row, V, L);
  const bool none = w.s == 0.0f, bad = w.s != w.s;
  const float unit = plain ? kLn2 : 1.0f, logS = none ? 0.0f : plain ? log2f(w.s) : logf(w.s);
  auto log_prob = [&](float x) { return fminf(((plain ? __builtin_fmaf(x, kLog2e, -w.m) : x - w.m) - logS) * unit, 0.0f); };
  if (tid == 0) {
    stg(a.lse + r, bad ? w.s : none ? -INFINITY : (w.m + logS) * unit);
    stg(a.entropy + r, bad ? w.s : none ? 0.0f : (logS - w.t / w.s) * unit);
  }
  // the given tokens under this row
  auto score = [&](int q) {
    const int t = ldg(a.tokens + q);
    float v = 0.0f;
    if (t >= V) v = NAN;
    else if (t >= 0) v = bad ? w.s : none ? -INFINITY : log_prob(value_at<BF16>(row, t));
    stg(a.logprob + q, v);
  };
  if (a.row_of == nullptr) {
    if (tid == 0 && r < a.m) score(r);
  } else {
    for (int q = tid; q < a.m; q += THREADS) {
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
    keep_best<THREADS>(L, count, k);
  } else {
    best_in_steps<BF16, THREADS>(row, V, k, L);
  }
  if (tid < k) {
    const uint64_t e = L.keep[tid];
    stg(a.top_token + (size_t)r * k + tid, e ? (int)~(uint32_t)e : -1);
    stg(a.top_logprob + (size_t)r * k + tid, bad ? w.s : e ? log_prob(unordered((uint32_t)(e >> 32))) : -INFINITY);
  }
}

}  // namespace

hipError_t launch_token_scores(const ScoresArgs& a, hipStream_t st) {
  // Up to a row per CU: 16 waves on each row; more rows: 8 waves, so that a CU
  // reads one row while it closes another.
  if (a.n <= 256) {
    if (a.bf16_in)
      scores_kernel<true, 1024><<<dim3(a.n), dim3(1024), 0, st>>>(a);
    else
      scores_kernel<false, 1024><<<dim3(a.n), dim3(1024), 0, st>>>(a);
  } else {
    if (a.bf16_in)
      scores_kernel<true, 512><<<dim3(a.n), dim3(512), 0, st>>>(a);
    else
      scores_kernel<false, 512><<<dim3(a.n), dim3(512), 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace llmcad
