// The answer side of a step of several requests: the adjustment of its logits
// rows (penalties for tokens that a row's own sequence holds, biases, masks), the
// greedy token of every row, and the walk of the requests' trees along them.
#include "batch.h"

namespace llmcad {

namespace {

constexpr int kThreads = 256;
constexpr int kWords = kAdjustChunk / 32;

// 16 bytes of logits at any element's alignment (one global load or store: they need
// no more than that on this GPU; a template's argument would lose the types' alignment).
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const f32x4u a = *(const LLMCAD_GLOBAL f32x4u*)p, b = *((const LLMCAD_GLOBAL f32x4u*)p + 1);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = a[e];
    x[4 + e] = b[e];
  }
}
__device__ __forceinline__ void load8(const bf16* p, float (&x)[8]) {
  const bf16x8u a = *(const LLMCAD_GLOBAL bf16x8u*)p;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = bf2f(a[e]);
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  f32x4u a, b;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    a[e] = x[e];
    b[e] = x[4 + e];
  }
  *(LLMCAD_GLOBAL f32x4u*)p = a;
  *((LLMCAD_GLOBAL f32x4u*)p + 1) = b;
}
__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
  bf16x8u a;
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = f2bf(x[e]);
  *(LLMCAD_GLOBAL bf16x8u*)p = a;
}
__device__ __forceinline__ float load1(const float* p) { return ldg(p); }
__device__ __forceinline__ float load1(const bf16* p) { return bf2f(ldg(p)); }
__device__ __forceinline__ void store1(float* p, float x) { stg(p, x); }
__device__ __forceinline__ void store1(bf16* p, float x) { stg(p, f2bf(x)); }
__device__ __forceinline__ float rounded(float x, const float*) { return x; }
__device__ __forceinline__ float rounded(float x, const bf16*) { return bf2f(f2bf(x)); }

// Order of a row's candidates in 64 bits: the value, then the lower token.  NaN is
// above all; -0 is 0.
__device__ __forceinline__ uint64_t best_key(float v, int token) {
  if (v != v) return ~0ull;
  const uint32_t u = __float_as_uint(v + 0.0f);
  return (uint64_t)(u >> 31 ? ~u : u | 0x80000000u) << 32 | (uint32_t)~token;
}
constexpr uint64_t kNone = (uint64_t)(~0xff800000u) << 32 | 0xffffffffu;  // -inf at token 0: nothing is above
__device__ __forceinline__ int best_token(uint64_t key) {
  return key == ~0ull || key <= kNone ? -1 : (int)~(uint32_t)key;
}
__device__ __forceinline__ uint64_t wave_best(uint64_t k) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)k, off, kWave);
    if (o > k) k = o;
  }
  return k;
}

// What a workgroup knows of its piece of the vocabulary: how often a token occurs in
// the answer so far, which ones occur at all, and which have a bias (the index of its
// last entry).
struct Marks {
  uint32_t count[kAdjustChunk];
  uint32_t bias[kAdjustChunk];  // entry + 1 of the request's list
  uint32_t seen[kWords];        // in the history
  uint32_t own[kWords];         // in the row's branch
  uint32_t biased[kWords];
  uint64_t best[kThreads / kWave];
};

__device__ __forceinline__ uint32_t byte_of(const uint32_t* words, int piece) { return ((const uint8_t*)words)[piece]; }

template <class T>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a) {
#pragma clang fp contract(off)
  __shared__ Marks m;
  if (!plan_is_for(a.head, a.B, a.N)) return;
  const int tid = threadIdx.x, chunk = blockIdx.x % a.chunks, base = chunk * kAdjustChunk;
  const int r0 = blockIdx.x / a.chunks * a.rows_per, r1 = r0 + a.rows_per < a.N ? r0 + a.rows_per : a.N;
  const int size = a.V - base < kAdjustChunk ? a.V - base : kAdjustChunk;
  const int words = (a.V + 31) / 32;
  int current = -1, answer0 = 0, bias0 = 0;
  bool active = false, listed = false;
  float rho = 1.0f, presence = 0.0f, frequency = 0.0f;
  BatchRequest q{};
  for (int r = r0; r < r1; ++r) {
    const int request = wave_uniform(ldg(a.row_req + r));
    if (request < 0) continue;
    constexpr int PIECES = kAdjustChunk / kThreads / 8;
    const T* in = (const T*)a.logits + (long long)r * a.stride + base;
    float x[PIECES][8];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int at = (p * kThreads + tid) * 8;
      if (at + 8 <= size) {
        load8(in + at, x[p]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[p][e] = at + e < size ? load1(in + at + e) : 0.0f;
      }
    }
    if (request != current) {
      if (current >= 0) lds_barrier();
      current = request;
      q = ldg(a.req + request);
      active = false;
      if (a.by.penalties) {
        rho = ldg(a.by.penalties + 3 * (size_t)request);
        presence = ldg(a.by.penalties + 3 * (size_t)request + 1);
        frequency = ldg(a.by.penalties + 3 * (size_t)request + 2);
        active = !(rho == 1.0f && presence == 0.0f && frequency == 0.0f);  // (1 and zeros change no value)
      }
      answer0 = a.by.prompt_len ? ldg(a.by.prompt_len + request) : 0;
      int bias1 = 0;
      bias0 = 0;
      if (a.by.bias_start) {
        bias0 = ldg(a.by.bias_start + request);
        bias1 = ldg(a.by.bias_start + request + 1);
        bias0 = bias0 < 0 ? 0 : bias0;
        bias1 = bias1 > a.by.n_bias ? a.by.n_bias : bias1;
      }
      listed = bias0 < bias1;
      if (active || listed) {
        for (int e = tid; e < kAdjustChunk / 4; e += kThreads) {
          ((uint4*)m.count)[e] = make_uint4(0, 0, 0, 0);
          if (listed) ((uint4*)m.bias)[e] = make_uint4(0, 0, 0, 0);
        }
        for (int e = tid; e < kWords; e += kThreads) m.seen[e] = m.own[e] = m.biased[e] = 0;
        lds_barrier();
        if (active && a.by.history) {
          const int* text = a.by.history + (long long)request * a.by.history_stride;
          const int len = q.held < a.by.history_stride ? q.held : (int)a.by.history_stride;
#pragma unroll 4
          for (int i = tid; i < len; i += kThreads) {
            const uint32_t t = (uint32_t)ldg(text + i) - (uint32_t)base;
            if (t < (uint32_t)size) {
              atomicOr(&m.seen[t >> 5], 1u << (t & 31));
              if (i >= answer0) atomicAdd(&m.count[t], 1u);
            }
          }
        }
        if (listed)
          for (int i = bias0 + tid; i < bias1; i += kThreads) {
            const uint32_t t = (uint32_t)ldg(a.by.bias_token + i) - (uint32_t)base;
            if (t < (uint32_t)size) {
              atomicOr(&m.biased[t >> 5], 1u << (t & 31));
              atomicMax(&m.bias[t], (uint32_t)(i - bias0) + 1);
            }
          }
      }
    }
    // the row's branch: its ancestors' tokens and its own
    int mine = -1;
    bool counted = false;
    if (active && tid < LLMCAD_MAX_NODES) {
      const uint4 w = ldg((const uint4*)(a.mask + (size_t)r * 4));
      const uint32_t word = tid < 64 ? (tid < 32 ? w.x : w.y) : (tid < 96 ? w.z : w.w);
      if (word >> (tid & 31) & 1) {
        const uint32_t t = (uint32_t)ldg(a.by.tokens + q.row0 + tid) - (uint32_t)base;
        if (t < (uint32_t)size) {
          int depth = __popc(word & ((1u << (tid & 31)) - 1));
          depth += (tid >= 32 ? __popc(w.x) : 0) + (tid >= 64 ? __popc(w.y) : 0) + (tid >= 96 ? __popc(w.z) : 0);
          mine = (int)t;
          counted = (long long)q.held + depth >= answer0;
          atomicOr(&m.own[t >> 5], 1u << (t & 31));
          if (counted) atomicAdd(&m.count[t], 1u);
        }
      }
    }
    if (active || listed) lds_barrier();
    const int state = a.by.allow && a.by.mask_of ? ldg(a.by.mask_of + r) : -1;
    const uint8_t* allow = state >= 0 && state < a.by.n_masks ? (const uint8_t*)(a.by.allow + (size_t)state * words) : nullptr;
    float best = -INFINITY;
    int best_at = 0;
    bool nan = false;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int at = (p * kThreads + tid) * 8;
      if (at >= size) continue;
      const int piece = at / 8, global = (base + at) / 8;
      uint32_t seen = 0, biased = 0, allowed = state < 0 ? 0xffu : 0u;
      if (allow) allowed = ldg(allow + global);
      if (active) {
        seen = byte_of(m.seen, piece) | byte_of(m.own, piece);
        if (a.by.seen) seen |= ldg((const uint8_t*)a.by.seen + global);
      }
      if (listed) biased = byte_of(m.biased, piece);
      if (seen | biased) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float v = x[p][e];
          if (seen >> e & 1) {
            const uint32_t c = m.count[at + e];
            v = v > 0.0f ? v / rho : v * rho;
            v = v - frequency * (float)c;
            v = v - (c > 0 ? presence : 0.0f);
          }
          if (biased >> e & 1) v = v + ldg(a.by.bias_value + bias0 + (m.bias[at + e] - 1));
          x[p][e] = v;
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[p][e] = rounded(allowed >> e & 1 ? x[p][e] : -INFINITY, (const T*)nullptr);
        if (at + e < size) {
          nan |= x[p][e] != x[p][e];
          if (x[p][e] > best) {
            best = x[p][e];
            best_at = at + e;
          }
        }
      }
      if (a.out) {
        T* out = (T*)a.out + (long long)r * a.out_stride + base + at;
        if (at + 8 <= size) {
          store8(out, x[p]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (at + e < size) store1(out + e, x[p][e]);
        }
      }
    }
    if (a.greedy) {
      const uint64_t k = wave_best(nan ? ~0ull : best_key(best, base + best_at));
      if ((tid & 63) == 0) m.best[tid >> 6] = k;
    }
    if (a.greedy || active) lds_barrier();  // (every wave is done with the row's marks)
    if (a.greedy && tid == 0) {
      uint64_t k = m.best[0];
      for (int w = 1; w < kThreads / kWave; ++w) k = m.best[w] > k ? m.best[w] : k;
      if (a.chunks > 1)
        stg(a.part + (size_t)r * a.chunks + chunk, k);
      else
        stg(a.greedy + r, best_token(k));
    }
    if (mine >= 0) {
      m.own[mine >> 5] = 0;
      if (counted) atomicSub(&m.count[mine], 1u);
    }
    if (a.greedy || active) lds_barrier();
  }
}

// The best of a row's pieces: a wave per row.
__global__ __launch_bounds__(kThreads) void greedy_kernel(AdjustArgs a) {
  const int r = blockIdx.x * (kThreads / kWave) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (!plan_is_for(a.head, a.B, a.N) || r >= a.N || ldg(a.row_req + r) < 0) return;
  uint64_t k = 0;
  for (int c = lane; c < a.chunks; c += kWave) {
    const uint64_t o = ldg(a.part + (size_t)r * a.chunks + c);
    if (o > k) k = o;
  }
  k = wave_best(k);
  if (lane == 0) stg(a.greedy + r, best_token(k));
}

// ---------------------------------------------------------------- accept walk
//
// A row is reached if the tokens of all its ancestors and its own (the root's apart) are
// the greedy tokens of their parents; its mask names them, and its parent is the last
// ancestor before it.  Of the deepest reached rows the first ends the walk, and the k-th
// bit of its mask is the k-th entry of the path.  A workgroup per request, one row per
// thread; bound by latency (a handful of dependent loads).
__global__ __launch_bounds__(LLMCAD_MAX_NODES) void accept_kernel(AcceptArgs a) {
  __shared__ uint64_t wrong_s[2];
  __shared__ int best_s[2];
  __shared__ uint32_t path_mask[4];
  if (!plan_is_for(a.head, a.B, a.N)) return;
  const int b = blockIdx.x, i = threadIdx.x, wave = i >> 6, lane = i & 63;
  const BatchRequest q = ldg(a.req + b);
  if (q.n == 0) {
    if (i == 0) stg(a.accept_len + b, -1);
    return;
  }
  uint32_t w[4] = {0, 0, 0, 0};
  bool wrong = false;
  if (i < q.n) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = ldg(a.mask + (size_t)(q.row0 + i) * 4 + j);
    int parent = -1;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t before = i >= 32 * (j + 1) ? w[j] : i > 32 * j ? w[j] & ((1u << (i - 32 * j)) - 1) : 0u;
      if (before) parent = 32 * j + 31 - __clz(before);
    }
    if (parent >= 0) {
      const int t = ldg(a.greedy + q.row0 + parent);
      wrong = t < 0 || t != ldg(a.tokens + q.row0 + i);
    }
  }
  const uint64_t any = __ballot(wrong);
  if (lane == 0) wrong_s[wave] = any;
  __syncthreads();
  int key = -1;
  if (i < q.n) {
    const uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
    if (!((lo & wrong_s[0]) | (hi & wrong_s[1])))
      key = (__popcll(lo) + __popcll(hi) - 1) * LLMCAD_MAX_NODES + (LLMCAD_MAX_NODES - 1 - i);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const int o = __shfl_xor(key, off, kWave);
    key = o > key ? o : key;
  }
  if (lane == 0) best_s[wave] = key;
  __syncthreads();
  const int best = best_s[0] > best_s[1] ? best_s[0] : best_s[1];
  const int depth = best / LLMCAD_MAX_NODES, last = LLMCAD_MAX_NODES - 1 - best % LLMCAD_MAX_NODES;  // (the root is always reached)
  if (i == last) {
#pragma unroll
    for (int j = 0; j < 4; ++j) path_mask[j] = w[j];
    stg(a.accept_len + b, depth);
    stg(a.next_token + b, ldg(a.greedy + q.row0 + last));
  }
  __syncthreads();
  if (i >= q.n) return;
  // thread j, if it is on the path, knows its place there: the path's rows before it
  const uint64_t lo = (uint64_t)path_mask[1] << 32 | path_mask[0], hi = (uint64_t)path_mask[3] << 32 | path_mask[2];
  if ((i < 64 ? lo >> i : hi >> (i - 64)) & 1) {
    const int k = i < 64 ? __popcll(lo & ((1ull << i) - 1)) : __popcll(lo) + __popcll(hi & ((1ull << (i - 64)) - 1));
    stg(a.path + q.row0 + k, i);
    if (a.history && (long long)q.held + k < a.history_stride)
      stg(a.history + (long long)b * a.history_stride + q.held + k, ldg(a.tokens + q.row0 + i));
  }
  if (i > depth) stg(a.path + q.row0 + i, -1);
}

}  // namespace

hipError_t launch_batch_adjust(const AdjustArgs& args, hipStream_t st) {
  AdjustArgs a = args;
  a.chunks = cdiv(a.V, kAdjustChunk);
  a.rows_per = 1;
  while ((size_t)a.chunks * cdiv(a.N, a.rows_per) >= 1u << 24) a.rows_per *= 2;  // (a launch takes 2^32 threads)
  const dim3 grid((unsigned)((size_t)a.chunks * cdiv(a.N, a.rows_per)));
  if (a.bf16_in)
    adjust_kernel<bf16><<<grid, dim3(kThreads), 0, st>>>(a);
  else
    adjust_kernel<float><<<grid, dim3(kThreads), 0, st>>>(a);
  if (a.greedy && a.chunks > 1) greedy_kernel<<<dim3(cdiv(a.N, kThreads / kWave)), dim3(kThreads), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_batch_accept(const AcceptArgs& a, hipStream_t st) {
  accept_kernel<<<dim3(a.B), dim3(LLMCAD_MAX_NODES), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace llmcad
