// Scores of logits rows: log probabilities of given tokens, the entropy, the
// normaliser and the most likely tokens.
//
// One pass over a row, the next tile's loads in flight while one is computed:
// every thread keeps the running maximum m of its values, the sum S of exp(x - m)
// and T of exp(x - m) (x - m), rescaled when m grows, in fp32 and in base 2 (one
// product less per value); joined over the workgroup, lse = m + log S and the
// entropy is log S - T / S.  A sum of 0 or NaN (nothing but -inf, a NaN, or values
// whose product with log2 e leaves fp32) is taken again in natural units.
//
// The k largest values come out of the same pass.  The first tile gives a lower
// bound of the k-th largest value: the k-th largest of 64 groups' maxima, of 256 for
// k above 32 (about as many values as k lie above it in the tile; always 256: 64.3 us
// for the 52.8 below).  Every 16-byte piece with a value from the bound on is held in
// LDS as it lies.  From time to time the held pieces' values join a list there, which
// is cut to its k best, and the k-th of them becomes the bound; at the end once more.
// The list is sorted by counting for each entry those above it.  A row whose pieces
// or list do not fit (values in rising order, say) is read once more in steps that
// cut the list back to its k best.
//
// Bound by the reads up to k of 32: 1024 bf16 rows of 128000 take 50.3 us without
// alternatives (5200 GB/s), 52.8 with 8 or 16, 56.3 with 32; 81 with 64, where the
// bound and the ranking, in which a row's workgroup reads nothing, are not hidden.
// fp32 rows with 20 take 94 us (5600 GB/s).
#include <algorithm>

#include "batch.h"

namespace llmcad {

namespace {

constexpr int kPieces = 4;  // 16-byte pieces of a row per thread and tile
constexpr int kHeld = 512;
constexpr int kList = 2048;
constexpr int kGroups = 256;
constexpr float kLowest = -3.402823466e38f;        // (finite: x - m stays a number for rows of -inf)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct ScoreLds {
  float m[16], s[16], t[16];  // by wave
  __align__(16) float group[kGroups];
  float bound;
  int pieces, count;
  __align__(16) uint32_t held[kHeld][4];  // 16-byte pieces of the row with a value from the bound on
  int held_at[kHeld];                     // the tokens of their first values
  __align__(16) uint64_t list[kList];  // ordered value bits << 32 | ~token: larger is better, ties to the lower token
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
// what lies outside [lo, hi) reads as -inf and is not touched.)
template <bool BF16, int THREADS>
struct Tile {
  static constexpr int N = BF16 ? 8 : 4;             // values per piece
  static constexpr int PER = N * kPieces;            // values per thread
  static constexpr int SIZE = PER * THREADS;
  u32x4 raw[kPieces];

  __device__ static __forceinline__ long at(long base, int piece) { return base + (long)N * (piece * THREADS + (int)threadIdx.x); }
  __device__ __forceinline__ void load(const char* row, long base, int lo, int hi) {
    constexpr int ES = 16 / N;
    if (base >= lo && base + SIZE <= hi) {
#pragma unroll
      for (int v = 0; v < kPieces; ++v) raw[v] = ldg((const u32x4*)(row + at(base, v) * ES));
      return;
    }
#pragma unroll
    for (int v = 0; v < kPieces; ++v) {
      const long i0 = at(base, v);
      const uint32_t none = BF16 ? 0xff80ff80u : 0xff800000u;
      u32x4 x = {none, none, none, none};
      if (i0 >= lo && i0 + N <= hi) {
        x = ldg((const u32x4*)(row + i0 * ES));
      } else if (i0 < hi) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const long i = i0 + e;
          if (i < lo || i >= hi) continue;
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
};

template <bool BF16>
__device__ __forceinline__ float value_at(const void* row, int i) {
  return BF16 ? bf2f(ldg((const bf16*)row + i)) : ldg((const float*)row + i);
}

// For each of the list's first count entries how many lie above it: to(entry, above).
// All threads call it, a barrier in front.  Groups of neighbouring lanes count for
// one entry together, in pieces of two entries, four reads in flight (one
// entry after another: 36 us more for the 64 best of 1024 bf16 rows of 128000).
template <int THREADS, typename TO>
__device__ __forceinline__ void rank(ScoreLds& L, int count, TO to) {
  typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));
  int share = kWave;  // lanes per entry
  while (share > 1 && count * share > THREADS) share >>= 1;
  const int part = threadIdx.x & (share - 1), round = 8 * share;
  const int end = (count + round - 1) / round * round;  // (at most kList)
  for (int j = count + threadIdx.x; j < end; j += THREADS) L.list[j] = 0;  // above no entry
  __syncthreads();
  for (int i0 = 0; i0 < count; i0 += THREADS / share) {
    const int i = i0 + threadIdx.x / share;
    const uint64_t mine = i < count ? L.list[i] : 0;
    int above = 0;
    for (int j = 0; j < end; j += round) {
      u64x2 o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = *(const u64x2*)&L.list[j + 2 * (e * share + part)];
#pragma unroll
      for (int e = 0; e < 4; ++e) above += (o[e].x > mine ? 1 : 0) + (o[e].y > mine ? 1 : 0);
    }
    for (int off = share >> 1; off >= 1; off >>= 1) above += __shfl_xor(above, off, kWave);
    if (i < count && part == 0) to(mine, above);
  }
  __syncthreads();
}

// The list's k best, sorted, in L.keep (0: no entry).  All threads call it.
template <int THREADS>
__device__ __forceinline__ void keep_best(ScoreLds& L, int count, int k) {
  if (threadIdx.x < k) L.keep[threadIdx.x] = 0;
  rank<THREADS>(L, count, [&](uint64_t entry, int above) {
    if (above < k) L.keep[above] = entry;
  });
}

// L.bound: the k-th largest of groups' maxima, groups of neighbouring threads (64
// of them for k up to 32: at most about 44 values of a tile lie above it then).
template <int THREADS>
__device__ __forceinline__ void first_bound(ScoreLds& L, float top, int k) {
  const int groups = k <= 32 ? 64 : kGroups, lanes = THREADS / groups, share = groups / lanes;
  float gm = top;
  for (int off = 1; off < lanes; off <<= 1) gm = fmaxf(gm, __shfl_xor(gm, off, kWave));
  const int group = threadIdx.x / lanes, part = threadIdx.x % lanes;
  if (part == 0) L.group[group] = gm;
  __syncthreads();
  int before = 0;  // the groups before this one, a share of them per lane
  for (int j = part * share; j < (part + 1) * share; j += 4) {
    const f32x4 o = *(const f32x4*)&L.group[j];
#pragma unroll
    for (int e = 0; e < 4; ++e) before += o[e] > gm || (o[e] == gm && j + e < group) ? 1 : 0;
  }
  for (int off = 1; off < lanes; off <<= 1) before += __shfl_xor(before, off, kWave);
  if (part == 0 && before == k - 1) L.bound = gm;
  __syncthreads();
}

// The held pieces' values from the bound on go to the list.  False if there were
// more than fit.  All threads call it.
template <bool BF16, int THREADS>
__device__ __forceinline__ bool list_pieces(ScoreLds& L, float bound) {
  constexpr int N = BF16 ? 8 : 4;
  __syncthreads();
  const int pieces = L.pieces;
  if (pieces > kHeld) return false;
  for (int j = threadIdx.x; j < pieces * N; j += THREADS) {
    const int e = j % N;
    const uint32_t w = L.held[j / N][BF16 ? e / 2 : e];
    const float x = __uint_as_float(!BF16 ? w : e & 1 ? w & 0xffff0000u : w << 16);
    if (!(x >= bound)) continue;
    const int at = atomicAdd(&L.count, 1);
    if (at < kList) L.list[at] = (uint64_t)ordered(x) << 32 | (uint32_t)~(uint32_t)(L.held_at[j / N] + e);
  }
  __syncthreads();
  return L.count <= kList;
}

// The k best of a row whose list overflowed.
template <bool BF16, int THREADS>
__device__ __attribute__((noinline)) void best_in_steps(const void* row, int lo, int hi, int k, ScoreLds& L) {
  uint64_t least = 0;  // the k-th best so far: later entries must be larger
  __syncthreads();
  if (threadIdx.x == 0) L.count = 0;
  for (long i0 = lo; i0 < hi; i0 += THREADS) {
    __syncthreads();
    const long i = i0 + threadIdx.x;
    if (i < hi) {
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

// What a row's log probabilities need: its maximum and the logarithm of its sum, in
// base 2 or natural units.
typedef f32x4 RowScore;  // (maximum, logarithm, kind)
enum { ROW_LOG2 = 0, ROW_NATURAL = 1, ROW_NONE = 2, ROW_BAD = 3 };
__device__ __forceinline__ float log_prob(const RowScore& s, float x) {
  const bool plain = s[2] == ROW_LOG2;
  const float unit = plain ? kLn2 : 1.0f;
  const float d = plain ? __builtin_fmaf(x, kLog2e, -s[0]) : x - s[0];
  if (d == -INFINITY) return x - s[0] * unit;  // (a finite value far below, in natural units)
  return fminf((d - s[1]) * unit, 0.0f);
}
// Given token q under its row.
template <bool BF16>
__device__ __forceinline__ void score_token(const ScoresArgs& a, int q, const char* row, const RowScore& s) {
  const int t = ldg(a.tokens + q);
  float v = 0.0f;
  if (t >= a.V) v = NAN;
  else if (t >= 0) v = s[2] == ROW_BAD ? NAN : s[2] == ROW_NONE ? -INFINITY : log_prob(s, value_at<BF16>(row, t));
  stg(a.logprob + q, v);
}

// The outputs of row r from its sums w (log2 domain).  All threads call it; best():
// the row's k best to L.keep.
template <bool BF16, int THREADS, typename BEST>
__device__ __forceinline__ void finish(const ScoresArgs& a, int r, const char* row, Sums w, ScoreLds& L, BEST best) {
  const int tid = threadIdx.x, V = a.V, k = a.k;
  // A sum of 0 or NaN: a row of nothing but -inf, with a NaN or +inf -- or with
  // values so large that their log2 is no fp32 number.
  const bool plain = w.s > 0.0f;
  if (!plain) w = sums_again<BF16, THREADS>(row, V, L);
  const bool none = w.s == 0.0f, bad = w.s != w.s;
  const float unit = plain ? kLn2 : 1.0f, logS = none ? 0.0f : plain ? log2f(w.s) : logf(w.s);
  const RowScore row_score = {w.m, logS, (float)(bad ? ROW_BAD : none ? ROW_NONE : plain ? ROW_LOG2 : ROW_NATURAL), 0.0f};
  if (tid == 0) {
    stg(a.lse + r, bad ? w.s : none ? -INFINITY : (w.m + logS) * unit);
    stg(a.entropy + r, bad ? w.s : none ? 0.0f : (logS - w.t / w.s) * unit);
  }
  // the given tokens under this row
  if (a.row_of == nullptr) {
    if (tid == 0 && r < a.m) score_token<BF16>(a, r, row, row_score);
  } else if (a.row_scores != nullptr) {
    if (tid == 0) stg((RowScore*)a.row_scores + r, row_score);
  } else {
    for (int q = tid; q < a.m; q += THREADS) {
      const int of = ldg(a.row_of + q);
      if (of == r) score_token<BF16>(a, q, row, row_score);
      else if (r == 0 && (of < 0 || of >= a.n)) stg(a.logprob + q, (float)NAN);
    }
  }
  if (k == 0) return;
  if (!bad) {
    best();
  } else if (tid < k) {
    L.keep[tid] = 0;  // (read by the same thread)
  }
  if (tid < k) {
    const uint64_t e = L.keep[tid];
    stg(a.top_token + (size_t)r * k + tid, e ? (int)~(uint32_t)e : -1);
    stg(a.top_logprob + (size_t)r * k + tid, bad ? w.s : e ? log_prob(row_score, unordered((uint32_t)(e >> 32))) : -INFINITY);
  }
}

// SPLIT: a workgroup per part of a row; sums and best values go to the workspace.
// (Four waves per SIMD: 133 registers leave three, 64 us for 58 with k of 20; the
// parts are a workgroup per CU.)
template <bool BF16, int THREADS, bool SPLIT>
__global__ __launch_bounds__(THREADS, SPLIT ? 2 : 4) void scores_kernel(ScoresArgs a) {
  typedef Tile<BF16, THREADS> T_;
  __shared__ ScoreLds L;
  constexpr int ESIZE = BF16 ? 2 : 4;
  const int r = SPLIT ? blockIdx.x / a.parts : blockIdx.x, part = SPLIT ? blockIdx.x % a.parts : 0, tid = threadIdx.x, k = a.k;
  const int lo = SPLIT ? part * a.span : 0, hi = SPLIT ? min(a.V, lo + a.span) : a.V;
  const char* row = (const char*)a.logits + (size_t)r * a.stride * ESIZE;
  // tiles start on the 16-byte boundary at or before the first value
  const long lead = (long)(((uintptr_t)(row + (size_t)lo * ESIZE) & 15) / ESIZE);
  if (tid == 0) {
    L.pieces = L.count = 0;
    L.bound = -INFINITY;
  }
  Sums w = {-1e37f, 0.0f, 0.0f};  // (in the log2 domain: one product less per value)
  float bound = -INFINITY;
  T_ tile, ahead;
  ahead.load(row, lo - lead, lo, hi);
  // The bound is raised after this many tiles, and again when they have doubled:
  // before many more than kHits values are held.  Each time costs about 1 us, which
  // a row alone on its CU waits for (31 fp32 rows of 90000, k of 8: 18.8 us with 128,
  // 20.1 with 32) and other rows' workgroups fill (1024 bf16 rows of 128000, k of 8:
  // 63.5 and 52.9; k of 32 59.7 and 56.4).
  constexpr int kHits = THREADS == 1024 ? 128 : 32;
  int done = 0, next = max(2, kHits / max(k, 1));
  bool listed = true;  // held pieces and list have had room so far
  for (long base = lo - lead; base < hi; base += T_::SIZE) {
    tile = ahead;
    if (base + T_::SIZE < hi) ahead.load(row, base + T_::SIZE, lo, hi);
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
        first_bound<THREADS>(L, top, k);
        bound = fmaxf(L.bound, kLowest);  // (-inf is no alternative)
      }
      int hits = 0;
#pragma unroll
      for (int v = 0; v < kPieces; ++v) hits += tops[v] >= bound ? 1 : 0;
      if (hits > 0) {
        int at = atomicAdd(&L.pieces, hits);
#pragma unroll
        for (int v = 0; v < kPieces; ++v) {
          if (!(tops[v] >= bound)) continue;
          if (at < kHeld) {
            *(u32x4*)L.held[at] = tile.raw[v];
            L.held_at[at] = (int)T_::at(base, v);
          }
          ++at;
        }
      }
      ++done;
      if (listed && done == next && base + T_::SIZE < hi) {
        next *= 2;
        listed = list_pieces<BF16, THREADS>(L, bound);
        const int count = L.count;
        if (listed && count >= k) {
          keep_best<THREADS>(L, count, k);
          if (tid < k) L.list[tid] = L.keep[tid];
          bound = unordered((uint32_t)(L.keep[k - 1] >> 32));
        }
        __syncthreads();  // (all have read the counts)
        if (listed && tid == 0) {
          L.pieces = 0;
          if (count >= k) L.count = k;
        }
        __syncthreads();
      }
    }
  }
  join<THREADS>(L, w, 1.0f);
  auto best = [&]() {
    if (listed && list_pieces<BF16, THREADS>(L, bound))
      keep_best<THREADS>(L, L.count, k);
    else
      best_in_steps<BF16, THREADS>(row, lo, hi, k, L);
  };
  if (!SPLIT) {
    finish<BF16, THREADS>(a, r, row, w, L, best);
    return;
  }
  if (tid == 0) stg((f32x4*)a.part_sums + blockIdx.x, f32x4{w.m, w.s, w.t, 0.0f});
  if (k == 0) return;
  best();
  if (tid < k) stg(a.part_best + (size_t)blockIdx.x * k + tid, L.keep[tid]);
}

// Many given tokens, each under its row: a thread per token.
template <bool BF16>
__global__ __launch_bounds__(256) void tokens_kernel(ScoresArgs a) {
  const int q = blockIdx.x * 256 + threadIdx.x;
  if (q >= a.m) return;
  const int r = ldg(a.row_of + q);
  if (r < 0 || r >= a.n)
    stg(a.logprob + q, (float)NAN);
  else
    score_token<BF16>(a, q, (const char*)a.logits + (size_t)r * a.stride * (BF16 ? 2 : 4), ldg((const RowScore*)a.row_scores + r));
}

// A workgroup per row joins its parts.
constexpr int kJoinThreads = 1024;
template <bool BF16>
__global__ __launch_bounds__(kJoinThreads) void scores_join_kernel(ScoresArgs a) {
  __shared__ ScoreLds L;
  const int r = blockIdx.x, tid = threadIdx.x, k = a.k, parts = a.parts, lane = tid & 63;
  const char* row = (const char*)a.logits + (size_t)r * a.stride * (BF16 ? 2 : 4);
  if (tid == 0) L.count = 0;
  Sums w = {-1e37f, 0.0f, 0.0f};
  if (tid < parts) {  // (parts <= a wave)
    const f32x4 p = ldg((const f32x4*)a.part_sums + r * parts + tid);
    w = Sums{p[0], p[1], p[2]};
  }
  const uint64_t* keys = a.part_best + (size_t)r * parts * k;
  uint64_t least = 0;
  if (k > 0) {
    // As many values as k lie at or above the largest of the parts' k-th best, and
    // at or above the least of their (k / parts)-th best.
    const int some = (k + parts - 1) / parts;
    uint64_t last = lane < parts ? ldg(keys + lane * k + k - 1) : 0, early = lane < parts ? ldg(keys + lane * k + some - 1) : ~0ull;
    for (int off = 32; off >= 1; off >>= 1) {
      const uint64_t l = __shfl_xor(last, off, kWave), e = __shfl_xor(early, off, kWave);
      last = l > last ? l : last;
      early = e < early ? e : early;
    }
    least = early > last ? early : last;
  }
  join<kJoinThreads>(L, w, 1.0f);  // (its barriers: the count is set)
  for (int j = tid; j < parts * k; j += kJoinThreads) {
    const uint64_t e = ldg(keys + j);
    if (e != 0 && e >= least) L.list[atomicAdd(&L.count, 1)] = e;
  }
  __syncthreads();
  finish<BF16, kJoinThreads>(a, r, row, w, L, [&]() { keep_best<kJoinThreads>(L, L.count, k); });
}

}  // namespace

// Up to 64 rows of many values: parts of about 16384, up to a workgroup per CU over
// all rows; their best values fit the list that joins them.  (The second launch
// costs 3 us of the host.  With k of 64, 31 fp32 rows of 250000 take 28.3 us, 40.2
// unsplit, one 23.2 and 37.9; with k of 8, 31 of 150000 21.4 and 23.0.  Rows of up to six
// such parts win nothing.  From 43 rows on the CUs allow five or four parts of longer
// rows, which pay all the same: with k of 8 on the GPU alone, 44 fp32 rows of 250000 20.9
// and 29.9, 64 of them 23.1 and 30.1, 44 and 64 of 100000 15.6 and 16.8, 17.1 and 17.0;
// 100 rows of 250000 take 38.0 and 33.3.)
int score_parts(int n, int V) {
  if (n > 64 || V <= 6 * 16384) return 1;
  return std::min({kList / LLMCAD_TOP_MAX, 256 / n, cdiv(V, 16384)});
}
static size_t part_bytes(int n, int parts, int k) {
  return parts > 1 ? align_up((size_t)n * parts * (sizeof(f32x4) + sizeof(uint64_t) * k), 16) : 0;
}
size_t score_work_bytes(int n, int V, int k) { return part_bytes(n, score_parts(n, V), k) + (size_t)n * sizeof(RowScore); }

// Tokens under rows of their own (row_of): up to this many, every row's workgroup
// looks through all of them; above, a second launch takes them.  The look grows
// with rows times tokens, the launch costs 2 to 3 us.  (us, looking / launching, bf16 rows and as
// many tokens: 31 of 32000 13.8 / 16.0, 1000 of 32000 16.5 / 18.6, 2000 of 32000 29.2 / 29.0, 4000 of
// 32000 54.6 / 47.7, of 2000 25.0 / 17.9, 20000 of 32000 594 / 231, 60000 of 8000 2749 / 222; 4000
// tokens under 31 rows 14.2 / 16.1.)
constexpr int kScanTokens = 2048;

template <bool BF16>
static void launch(const ScoresArgs& a, hipStream_t st) {
  // More rows than CUs: smaller workgroups, so that several rows share a CU and one
  // is read while another ranks its values (1024 bf16 rows of 128000, k of 8: 52.9 us
  // with 256 threads, 57.8 with 512; 2000 of 32000 44 and 49; 400 rows 45.8 and 37.4,
  // as a CU then has too few waves).
  if (a.parts > 1) {
    scores_kernel<BF16, 512, true><<<dim3(a.n * a.parts), dim3(512), 0, st>>>(a);
    scores_join_kernel<BF16><<<dim3(a.n), dim3(kJoinThreads), 0, st>>>(a);
  } else if (a.n <= 256) {
    scores_kernel<BF16, 1024, false><<<dim3(a.n), dim3(1024), 0, st>>>(a);
  } else if (a.n <= 512) {
    scores_kernel<BF16, 512, false><<<dim3(a.n), dim3(512), 0, st>>>(a);
  } else {
    scores_kernel<BF16, 256, false><<<dim3(a.n), dim3(256), 0, st>>>(a);
  }
  if (a.row_scores != nullptr) tokens_kernel<BF16><<<dim3(cdiv(a.m, 256)), dim3(256), 0, st>>>(a);
}

hipError_t launch_token_scores(ScoresArgs a, void* workspace, hipStream_t st) {
  a.parts = score_parts(a.n, a.V);
  a.span = cdiv(cdiv(a.V, a.parts), 64) * 64;
  a.part_sums = (float*)workspace;
  a.part_best = (uint64_t*)((f32x4*)workspace + (size_t)a.n * a.parts);
  a.row_scores = a.row_of != nullptr && a.m > kScanTokens ? (float*)((char*)workspace + part_bytes(a.n, a.parts, a.k)) : nullptr;
  if (a.bf16_in)
    launch<true>(a, st);
  else
    launch<false>(a, st);
  return hipGetLastError();
}

}  // namespace llmcad
