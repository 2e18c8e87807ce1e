// The answer side of a step of several requests: the adjustment of its logits
// rows (penalties for tokens that a row's own sequence holds, biases, masks), the
// greedy token of every row, and the walk of the requests' trees along them.
//
// A logit changes where its token occurs in the row's text, has a bias or is masked; the
// others are copied.  A workgroup takes pieces of 4096 tokens: it counts the text's tokens
// in a piece in LDS (4 bytes per token; integer atomics, whose order changes nothing), marks
// those that occur in a bitmap, and streams the piece, eight tokens a thread, adjusting
// the marked ones one after the other.  Every operation is a single fp32 one in the stated
// order, so that nothing depends on how rows are shared; each wave leaves its best token,
// and a second launch joins a row's.
//
// Bytes bound it where little is marked: 255 rows of 128000 bf16 logits are copied in 24 us
// (5300 GB/s) and their greedy tokens found in 15 (4300).  With all adjustments they take
// 45: the marked tokens (a tenth of a piece where a text's tokens are near each other) are
// taken by each lane from its own eight, so that a wave makes as many steps of about 60 vector
// instructions as its fullest lane has (three or four, where the mean is 0.8); a barrier waits
// for the slowest wave, and three workgroups are on a CU (LDS).  That is this loop's price and
// no limit: marked tokens dealt to all lanes of a wave have not been tried.  561 rows of 32000 fp32 logits take 27.6 us (14 to read
// them), a tree of 31 7.2, two launches' latency.
//
// Measured and left out: the next tile's loads in flight while one is computed (registers
// cost more waves than it hides: 27.6 -> 28.6; with two tiles in turn 40); the branch's tokens
// in registers instead of LDS, without barriers between rows (30.0 -> 30.6); two marked
// tokens at a time (41.5 -> 43.0); pieces of 2048 (41 -> 43.7 with long histories); 2 KB more
// LDS (two workgroups on a CU instead of three: 47 -> 61).
#include "batch.h"

namespace llmcad {

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;
constexpr int kWords = kAdjustChunk / 32;
static_assert(kThreads == kAdjustThreads && kAdjustChunk == 8 * kThreads && LLMCAD_MAX_NODES <= kThreads, "eight tokens of a piece, a row of a request per thread");

// 16 bytes of logits at any element's alignment (one global load or store: they need
// no more than that on this GPU; a template's argument would lose the types' alignment).
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));

// Eight of a row's logits as they lie.  What is behind the row's end is -inf.
template <class T>
struct Eight;
template <>
struct Eight<float> {
  f32x4u a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *(const LLMCAD_GLOBAL f32x4u*)p;
    b = *((const LLMCAD_GLOBAL f32x4u*)p + 1);
  }
  __device__ __forceinline__ void load(const float* p, int n) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a[e] = e < n ? ldg(p + e) : -INFINITY;
      b[e] = 4 + e < n ? ldg(p + 4 + e) : -INFINITY;
    }
  }
  __device__ __forceinline__ float get(int e) const { return e < 4 ? a[e] : b[e - 4]; }
  __device__ __forceinline__ void set(int e, float x) {
    if (e < 4) a[e] = x;
    else b[e - 4] = x;
  }
  __device__ __forceinline__ void store(float* p) const {
    *(LLMCAD_GLOBAL f32x4u*)p = a;
    *((LLMCAD_GLOBAL f32x4u*)p + 1) = b;
  }
  __device__ __forceinline__ void store(float* p, int n) const {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) stg(p + e, get(e));
  }
  static __device__ __forceinline__ float rounded(float x) { return x; }
};
template <>
struct Eight<bf16> {
  bf16x8u a;
  __device__ __forceinline__ void load(const bf16* p) { a = *(const LLMCAD_GLOBAL bf16x8u*)p; }
  __device__ __forceinline__ void load(const bf16* p, int n) {
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = e < n ? ldg(p + e) : (bf16)-INFINITY;
  }
  __device__ __forceinline__ float get(int e) const { return bf2f(a[e]); }
  __device__ __forceinline__ void set(int e, float x) { a[e] = f2bf(x); }
  __device__ __forceinline__ void store(bf16* p) const { *(LLMCAD_GLOBAL bf16x8u*)p = a; }
  __device__ __forceinline__ void store(bf16* p, int n) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bf16 x = a[e];
      if (e < n) stg(p + e, x);
    }
  }
  static __device__ __forceinline__ float rounded(float x) { return bf2f(f2bf(x)); }
};

// Order of a row's candidates in 64 bits: the value, then the lower token.  NaN is
// above all; -0 is 0.
__device__ __forceinline__ uint64_t best_key(float v, int token) {
  const uint32_t u = __float_as_uint(v + 0.0f);
  return v != v ? ~0ull : (uint64_t)(u >> 31 ? ~u : u | 0x80000000u) << 32 | (uint32_t)~token;
}
constexpr uint64_t kNone = (uint64_t)(~0xff800000u) << 32 | 0xffffffffu;  // -inf at token 0: nothing is above
__device__ __forceinline__ int best_token(uint64_t key) { return key == ~0ull || key <= kNone ? -1 : (int)~(uint32_t)key; }

// What a workgroup knows of its piece of the vocabulary: how often a token occurs in
// the answer so far, which ones occur at all, and which have a bias (the index of its
// last entry).
template <bool TEXT, bool BIAS>
struct Marks {
  uint32_t count[TEXT ? kAdjustChunk : 4];
  uint32_t bias[BIAS ? kAdjustChunk : 4];  // entry + 1 of the request's list
  uint32_t seen[kWords];                   // in the history
  uint32_t own[2][kWords];                 // in the row's branch (while one row's is cleared the next one's fills)
  uint32_t biased[kWords];
};

__device__ __forceinline__ uint32_t byte_of(const uint32_t* words, int piece) { return ((const uint8_t*)words)[piece]; }

// Tokens of the history in a workgroup's pieces, where it has several, piece by piece and
// counted within it; those whose occurrence counts have the top bit.
constexpr int kKept = 8192, kKeptPieces = 64;
struct Kept {
  uint16_t token[kKept];
  int start[kKeptPieces + 1];  // of each piece's; the last: of all (more than kKept: the history itself is read for every piece)
  int at[kKeptPieces];
};

// What is the same for all rows of a request.
struct Request {
  float rho, presence, frequency;
  bool active, listed;  // has penalties, has biases
  int row0, n, held, answer0;
  const int* text;  // its history, `len` tokens
  uint32_t len;     // (loops of a workgroup's steps past 2^31 - 1 stay in range unsigned)
  int bias0;
  uint32_t biases;
};

template <bool TEXT, bool BIAS>
__device__ __forceinline__ Request request_of(const AdjustArgs& a, int request) {
  Request q{};
  if (TEXT) {
    const float* p = a.by.penalties + 3 * (size_t)request;
    q.rho = ldg(p);
    q.presence = ldg(p + 1);
    q.frequency = ldg(p + 2);
    const BatchRequest* b = a.req + request;
    q.row0 = ldg(&b->row0);
    q.n = ldg(&b->n);
    q.held = ldg(&b->held);
    q.answer0 = a.by.prompt_len ? ldg(a.by.prompt_len + request) : 0;
    q.active = !(q.rho == 1.0f && q.presence == 0.0f && q.frequency == 0.0f);  // (1 and zeros change no value)
    q.text = a.by.history + (long long)request * a.by.history_stride;
    q.len = !q.active || !a.by.history ? 0 : (uint32_t)(q.held < a.by.history_stride ? q.held : a.by.history_stride);
  }
  if (BIAS) {
    int lo = ldg(a.by.bias_start + request), hi = ldg(a.by.bias_start + request + 1);
    lo = lo < 0 ? 0 : lo;
    hi = hi > a.by.n_bias ? a.by.n_bias : hi;
    q.bias0 = lo;
    q.biases = hi > lo ? (uint32_t)(hi - lo) : 0;
    q.listed = hi > lo;
  }
  return q;
}

// Sorts the tokens of the history in pieces first, first + step, ... by their piece (at
// most kKeptPieces): counted once, placed in a second pass.
__device__ __forceinline__ void keep_history(Kept& k, const Request& q, int vocab, int first, int step) {
  const int tid = threadIdx.x;
  constexpr int AHEAD = 8;  // loads in flight; so many are not read again for the second pass
  const float inverse = 1.0f / (float)step;
  const auto load = [&](int (&id)[AHEAD], uint32_t i0) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const uint32_t i = i0 + j * kThreads + tid;
      id[j] = i < q.len ? ldg(q.text + i) : -1;
    }
  };
  // f(which of the workgroup's pieces, j) for those of the ids that lie in one
  const auto each = [&](const int (&id)[AHEAD], auto f) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if ((uint32_t)id[j] >= (uint32_t)vocab) continue;
      const int c = id[j] / kAdjustChunk - first, piece = (int)(((float)c + 0.5f) * inverse);  // (at most 2^12: exact)
      if (c >= 0 && piece * step == c) f(piece, j);
    }
  };
  int head[AHEAD], more[AHEAD];
  load(head, 0);
  if (tid < kKeptPieces) k.at[tid] = 0;
  lds_barrier();
  const auto count = [&](int piece, int) { atomicAdd(&k.at[piece], 1); };
  each(head, count);
  for (uint32_t i0 = AHEAD * kThreads; i0 < q.len; i0 += AHEAD * kThreads) {
    load(more, i0);
    each(more, count);
  }
  lds_barrier();
  if (tid < kKeptPieces) {  // (one wave)
    const int mine = k.at[tid];
    int sum = mine;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const int o = __shfl_up(sum, off, kWave);
      if (tid >= off) sum += o;
    }
    k.start[tid + 1] = sum;
    k.at[tid] = sum - mine;
    if (tid == 0) k.start[0] = 0;
  }
  lds_barrier();
  if (k.start[kKeptPieces] > kKept) return;
  const auto place = [&](const int (&id)[AHEAD], uint32_t i0) {
    each(id, [&](int piece, int j) {
      k.token[atomicAdd(&k.at[piece], 1)] = (uint16_t)(id[j] % kAdjustChunk | ((int)(i0 + j * kThreads + tid) >= q.answer0 ? 0x8000 : 0));
    });
  };
  place(head, 0);
  for (uint32_t i0 = AHEAD * kThreads; i0 < q.len; i0 += AHEAD * kThreads) {
    load(more, i0);
    place(more, i0);
  }
}
static_assert(kKeptPieces == kWave, "a lane per piece");

// Clears the marks and makes those of the history and the biases in a piece; entry: the
// thread's of the bias list.
template <bool TEXT, bool BIAS>
__device__ __forceinline__ void mark_piece(const AdjustArgs& a, Marks<TEXT, BIAS>& m, const Request& q, const Kept* kept, int piece, int entry, int base, int size) {
  const int tid = threadIdx.x;
  constexpr int PER = kAdjustChunk / 4 / kThreads;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (TEXT && q.active) ((uint4*)m.count)[tid + i * kThreads] = make_uint4(0, 0, 0, 0);
    if (BIAS && q.listed) ((uint4*)m.bias)[tid + i * kThreads] = make_uint4(0, 0, 0, 0);
  }
  if (tid < kWords) m.seen[tid] = m.own[0][tid] = m.own[1][tid] = m.biased[tid] = 0;
  lds_barrier();
  if (TEXT && q.active) {
    const auto mark = [&](uint32_t id, bool counts) {
      const uint32_t t = id - (uint32_t)base;
      if (t < (uint32_t)size) {
        atomicOr(&m.seen[t >> 5], 1u << (t & 31));
        if (counts) atomicAdd(&m.count[t], 1u);
      }
    };
    if (kept && kept->start[kKeptPieces] <= kKept) {
      for (int i = kept->start[piece] + tid; i < kept->start[piece + 1]; i += kThreads) mark(base + (kept->token[i] & 0x7fffu), kept->token[i] >> 15);
    } else {
#pragma unroll 4
      for (uint32_t i = tid; i < q.len; i += kThreads) mark((uint32_t)ldg(q.text + i), (int)i >= q.answer0);
    }
  }
  if (BIAS && q.listed) {
    const auto mark = [&](int id, uint32_t i) {
      const uint32_t t = (uint32_t)id - (uint32_t)base;
      if (t < (uint32_t)size) {
        atomicOr(&m.biased[t >> 5], 1u << (t & 31));
        atomicMax(&m.bias[t], i + 1);
      }
    };
    mark(entry, tid);
    for (uint32_t i = tid + kThreads; i < q.biases; i += kThreads) mark(ldg(a.by.bias_token + q.bias0 + i), i);
  }
}

// The thread's entry of the request's bias list: its token.
template <bool BIAS>
__device__ __forceinline__ int entry_of(const AdjustArgs& a, const Request& q) {
  return BIAS && threadIdx.x < q.biases ? ldg(a.by.bias_token + q.bias0 + threadIdx.x) : -1;
}

// The thread's token of a row's branch, if there is one in the piece: marks it.
template <bool TEXT, bool BIAS>
struct Own {
  int at = -1;
  bool counted = false;
  __device__ __forceinline__ void mark(Marks<TEXT, BIAS>& m, int turn, const Request& q, int token, u32x4 branch, int base, int size) {
    const int tid = threadIdx.x;
    const uint32_t word = tid < 64 ? (tid < 32 ? branch.x : branch.y) : (tid < 96 ? branch.z : branch.w);
    const uint32_t t = (uint32_t)token - (uint32_t)base;
    at = -1;
    if (tid < LLMCAD_MAX_NODES && (word >> (tid & 31) & 1) && t < (uint32_t)size) {
      int depth = __popc(word & ((1u << (tid & 31)) - 1));
      depth += (tid >= 32 ? __popc(branch.x) : 0) + (tid >= 64 ? __popc(branch.y) : 0) + (tid >= 96 ? __popc(branch.z) : 0);
      at = (int)t;
      counted = (long long)q.held + depth >= q.answer0;
      atomicOr(&m.own[turn][t >> 5], 1u << (t & 31));
      if (counted) atomicAdd(&m.count[t], 1u);
    }
  }
  __device__ __forceinline__ void unmark(Marks<TEXT, BIAS>& m, int turn) const {
    if (at < 0) return;
    m.own[turn][at >> 5] = 0;
    if (counted) atomicSub(&m.count[at], 1u);
  }
};

// A thread's best of a row so far; NaN stays.
struct Best {
  float value = -INFINITY;
  int token = 0;
  __device__ __forceinline__ void join(const float (&x)[8], int first) {
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = __builtin_elementwise_maximum(top, x[e]);
    if (!(top <= value)) {
      int e0 = 7;
#pragma unroll
      for (int e = 6; e >= 0; --e) e0 = x[e] == top ? e : e0;
      token = first + e0;
      value = __builtin_elementwise_maximum(value, top);
    }
  }
  // The wave's best, to lane 0's partial result: the largest value, then the lowest of its tokens.
  __device__ __forceinline__ void write(uint64_t* part) const {
    const bool nan = __ballot(value != value) != 0;
    float top = value;
    top = fmaxf(top, dpp_f<kDppQuadXor1>(top));
    top = fmaxf(top, dpp_f<kDppQuadXor2>(top));
    top = fmaxf(top, dpp_f<kDppRowHalfMirror>(top));
    top = fmaxf(top, dpp_f<kDppRowMirror>(top));
    top = col4_max(top);
    int at = value == top ? token : 0x7fffffff;
    at = min(at, dpp_i<kDppQuadXor1>(at));
    at = min(at, dpp_i<kDppQuadXor2>(at));
    at = min(at, dpp_i<kDppRowHalfMirror>(at));
    at = min(at, dpp_i<kDppRowMirror>(at));
    float a, b;
    pair_xor16(__int_as_float(at), a, b);
    at = min(__float_as_int(a), __float_as_int(b));
    pair_xor32(__int_as_float(at), a, b);
    at = min(__float_as_int(a), __float_as_int(b));
    if ((threadIdx.x & 63) == 0) stg(part, nan ? (uint64_t)~0ull : best_key(top, at));
  }
};

// The eight logits of a thread, adjusted: in x, and rounded in f.
template <class T, bool TEXT, bool BIAS>
__device__ __forceinline__ void adjust_eight(const AdjustArgs& a, const Marks<TEXT, BIAS>& m, int turn, const Request& q, Eight<T>& x,
                                             float (&f)[8], uint32_t allowed, uint32_t prefix, int size) {
#pragma clang fp contract(off)
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = x.get(e);
  uint32_t seen = 0, biased = 0;
  if (TEXT && q.active) {
    // (The last word's bits that are no tokens are left out: of their -inf a penalty could make NaN or +inf.
    // Here, not at the load, which nothing should wait for: 45.6 us for 48.8 at 255 rows of 128000.)
    const int past = 8 * (int)threadIdx.x + 8 - size;  // (from 8 on the byte is 0)
    prefix &= 0xffu >> ((past > 0 ? past : 0) & 31);
    seen = (byte_of(m.seen, threadIdx.x) | byte_of(m.own[turn], threadIdx.x) | prefix) & allowed;
  }
  if (BIAS && q.listed) biased = byte_of(m.biased, threadIdx.x) & allowed;
  if (TEXT || BIAS) {
    // (few of a wave's tokens are touched: one after the other)
    for (uint32_t touched = seen | biased; touched; touched &= touched - 1) {
      const int i = __ffs(touched) - 1;
      float v = f[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) v = i == e ? f[e] : v;
      if (TEXT && (seen >> i & 1)) {
        const uint32_t n = m.count[8 * threadIdx.x + i];
        v = v > 0.0f ? v / q.rho : v * q.rho;
        v = v - q.frequency * (float)n;
        v = v - (n > 0 ? q.presence : 0.0f);
      }
      if (BIAS && (biased >> i & 1)) v = v + ldg(a.by.bias_value + q.bias0 + (m.bias[8 * threadIdx.x + i] - 1));
      v = Eight<T>::rounded(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = i == e ? v : f[e];
    }
  }
  const bool masked = allowed != 0xffu;
  if (__ballot(masked)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = allowed >> e & 1 ? f[e] : -INFINITY;
  }
  if (a.out && __ballot(masked || (seen | biased) != 0)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x.set(e, f[e]);
  }
}

template <class T>
__device__ __forceinline__ void load_eight(Eight<T>& x, const T* row, int base, int size) {
  const int at = 8 * threadIdx.x;
  if (at + 8 <= size)
    x.load(row + base + at);
  else
    x.load(row + base + at, size - at);
}
template <class T>
__device__ __forceinline__ void store_eight(const Eight<T>& x, T* row, int base, int size) {
  const int at = 8 * threadIdx.x;
  if (at + 8 <= size)
    x.store(row + base + at);
  else
    x.store(row + base + at, size - at);
}
// The thread's byte of a mask (bytes past the vocabulary's words are not read).
__device__ __forceinline__ uint32_t mask_byte(const uint32_t* words, int base, int size) {
  return 8 * (int)threadIdx.x < size ? ldg((const uint8_t*)words + base / 8 + threadIdx.x) : 0u;
}
__device__ __forceinline__ uint32_t allowed_byte(const AdjustArgs& a, int state, int base, int size) {
  if (state < 0) return 0xffu;
  return state < a.by.n_masks ? mask_byte(a.by.allow + (size_t)state * ((a.V + 31) / 32), base, size) : 0u;
}

// Where requests have several rows: a workgroup takes one piece of rows [r0, r1).  A
// request's marks are made once.
template <class T, bool TEXT, bool BIAS>
__global__ __launch_bounds__(kThreads, 6) void adjust_rows_kernel(AdjustArgs a) {
  __shared__ Marks<TEXT, BIAS> m;
  const int tid = threadIdx.x, lane = tid & 63, c = blockIdx.x % a.chunks, base = c * kAdjustChunk;
  const int size = a.V - base < kAdjustChunk ? a.V - base : kAdjustChunk;
  const int r0 = blockIdx.x / a.chunks * a.rows_per, r1 = r0 + a.rows_per < a.N ? r0 + a.rows_per : a.N;
  // (a lane for each of the workgroup's rows, at most 64)
  const int mine = r0 + lane < r1 ? r0 + lane : r1 - 1;
  const int requests = ldg(a.row_req + mine), states = a.by.mask_of ? ldg(a.by.mask_of + mine) : -1;
  if (!plan_is_for(a.head, a.B, a.N)) return;
  const T* logits = (const T*)a.logits;
  uint32_t prefix = 0;
  if (TEXT && a.by.seen) prefix = mask_byte(a.by.seen, base, size);
  int turn = 0;
  for (int r = r0; r < r1;) {
    // the rows of one request
    const int request = __builtin_amdgcn_readlane(requests, r - r0), first = r;
    const uint64_t others = __ballot(requests != request || r0 + lane >= r1) >> (r - r0);
    r = others ? r + __ffsll((unsigned long long)others) - 1 : r1;
    if (request < 0) continue;
    const Request q = request_of<TEXT, BIAS>(a, request);
    const bool marked = (TEXT && q.active) || (BIAS && q.listed);
    int token = -1;
    if (TEXT && q.active && tid < q.n) token = ldg(a.by.tokens + q.row0 + tid);  // (at most 128)
    if (marked) mark_piece<TEXT, BIAS>(a, m, q, nullptr, 0, entry_of<BIAS>(a, q), base, size);
    for (int row = first; row < r; ++row) {
      u32x4 branch = {0, 0, 0, 0};
      if (TEXT && q.active) branch = ldg((const u32x4*)(a.mask + (size_t)row * 4));
      Eight<T> x;
      load_eight(x, logits + (long long)row * a.stride, base, size);
      const uint32_t allowed = allowed_byte(a, __builtin_amdgcn_readlane(states, row - r0), base, size);
      Own<TEXT, BIAS> own;
      if (TEXT && q.active) own.mark(m, turn, q, token, branch, base, size);
      if ((TEXT && q.active) || (marked && row == first)) lds_barrier();
      float f[8];
      adjust_eight<T, TEXT, BIAS>(a, m, turn, q, x, f, allowed, prefix, size);
      if (a.out) store_eight(x, (T*)a.out + (long long)row * a.out_stride, base, size);
      if (a.greedy) {
        Best best;
        best.join(f, base + 8 * tid);
        best.write(a.part + ((size_t)row * a.chunks + c) * kWaves + tid / kWave);
      }
      if (TEXT && q.active) {
        lds_barrier();  // (every wave is done with the row's marks)
        own.unmark(m, turn);
        turn ^= 1;
      }
    }
    if (marked) lds_barrier();  // (the next request's marks begin with clear ones)
  }
}

// Where they have few: a workgroup takes every a.segments-th piece of one row (tokens
// that a text repeats lie near each other in many vocabularies).  The row's text is read
// once and sorted by piece (38 us for 41 where every piece goes through all of it).
template <class T, bool TEXT, bool BIAS>
__global__ __launch_bounds__(kThreads, 6) void adjust_row_kernel(AdjustArgs a) {
  __shared__ Marks<TEXT, BIAS> m;
  __shared__ Kept kept;
  const int tid = threadIdx.x, segment = blockIdx.x % a.segments, row = blockIdx.x / a.segments;
  const int c0 = segment, step = a.segments;
  const int request = wave_uniform(ldg(a.row_req + row)), state = a.by.mask_of ? wave_uniform(ldg(a.by.mask_of + row)) : -1;
  const T* logits = (const T*)a.logits + (long long)row * a.stride;
  auto size_of = [&](int c) { return a.V - c * kAdjustChunk < kAdjustChunk ? a.V - c * kAdjustChunk : kAdjustChunk; };
  if (request < 0 || !plan_is_for(a.head, a.B, a.N)) return;
  const Request q = request_of<TEXT, BIAS>(a, request);
  const bool marked = (TEXT && q.active) || (BIAS && q.listed);
  const bool sorted = q.len > 0 && step < a.chunks && a.chunks_per <= kKeptPieces;
  const int entry = entry_of<BIAS>(a, q);
  int token = -1;
  u32x4 branch = {0, 0, 0, 0};
  if (TEXT && q.active) {
    if (tid < q.n) token = ldg(a.by.tokens + q.row0 + tid);
    branch = ldg((const u32x4*)(a.mask + (size_t)row * 4));
    if (sorted) keep_history(kept, q, a.V, c0, step);
  }
  Best best;
  for (int c = c0, piece = 0; c < a.chunks; c += step, ++piece) {
    const int base = c * kAdjustChunk, size = size_of(c);
    Eight<T> x;
    load_eight(x, logits, base, size);
    const uint32_t allowed = allowed_byte(a, state, base, size), prefix = TEXT && a.by.seen ? mask_byte(a.by.seen, base, size) : 0u;
    if (marked) {
      mark_piece<TEXT, BIAS>(a, m, q, sorted ? &kept : nullptr, piece, entry, base, size);
      Own<TEXT, BIAS> own;
      if (TEXT && q.active) own.mark(m, 0, q, token, branch, base, size);
      lds_barrier();
    }
    float f[8];
    adjust_eight<T, TEXT, BIAS>(a, m, 0, q, x, f, allowed, prefix, size);
    if (a.out) store_eight(x, (T*)a.out + (long long)row * a.out_stride, base, size);
    if (a.greedy) best.join(f, base + 8 * tid);
    if (marked) lds_barrier();  // (the next piece's marks begin with clear ones)
  }
  if (a.greedy) best.write(a.part + ((size_t)row * a.segments + segment) * kWaves + tid / kWave);
}

// The best of a row's parts: a wave per row.
__global__ __launch_bounds__(256) void greedy_kernel(AdjustArgs a) {
  const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= a.N) return;
  const int request = ldg(a.row_req + r), parts = a.segments * kWaves;
  uint64_t k = 0;
  for (int c = lane; c < parts; c += kWave) {  // (of a row without a request: whatever lies there)
    const uint64_t o = ldg(a.part + (size_t)r * parts + c);
    if (o > k) k = o;
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    const uint64_t o = __shfl_xor((unsigned long long)k, off, kWave);
    if (o > k) k = o;
  }
  if (request < 0 || !plan_is_for(a.head, a.B, a.N)) return;
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

namespace {

template <class T, bool TEXT, bool BIAS>
void launch_adjust(const AdjustArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)((long long)a.segments * cdiv(a.N, a.rows_per)));
  if (a.chunks_per == 0)
    adjust_rows_kernel<T, TEXT, BIAS><<<grid, dim3(kThreads), 0, st>>>(a);
  else
    adjust_row_kernel<T, TEXT, BIAS><<<grid, dim3(kThreads), 0, st>>>(a);
}
template <class T>
void launch_adjust(const AdjustArgs& a, hipStream_t st) {
  if (a.by.penalties)
    a.by.bias_start ? launch_adjust<T, true, true>(a, st) : launch_adjust<T, true, false>(a, st);
  else
    a.by.bias_start ? launch_adjust<T, false, true>(a, st) : launch_adjust<T, false, false>(a, st);
}

}  // namespace

hipError_t launch_batch_adjust(const AdjustArgs& args, hipStream_t st) {
  AdjustArgs a = args;
  a.chunks = cdiv(a.V, kAdjustChunk);
  // About as many workgroups as the GPU holds (three on a CU, four without penalties): of
  // several rows each where requests have eight or more (32 trees of up to 41 with histories
  // of up to 1000: 27.6 us for 32.3), of several pieces of a row otherwise (four rows each
  // of 64 requests: 20.3 for 21.8; at eight each takes 40).  N counts padding and B requests
  // that sit out (the device alone knows the others): single tokens in a step sized for trees
  // take the first form, with the same results.
  const long long tiles = (long long)a.chunks * a.N;
  const bool rows = a.N >= 8ll * a.B && tiles < 1ll << 26;  // (a launch takes 2^32 threads)
  const long long want = a.by.penalties ? 768 : 1024;
  const int per = tiles < want ? 1 : (int)((tiles + want / 2) / want);
  a.rows_per = 1;
  a.chunks_per = 0;
  if (rows)
    a.rows_per = per < 16 ? per : 16;
  else
    a.chunks_per = per < a.chunks ? per : a.chunks;
  a.segments = a.chunks_per == 0 ? a.chunks : cdiv(a.chunks, a.chunks_per);
  if (a.bf16_in)
    launch_adjust<bf16>(a, st);
  else
    launch_adjust<float>(a, st);
  if (a.greedy) greedy_kernel<<<dim3(cdiv(a.N, 4)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_batch_accept(const AcceptArgs& a, hipStream_t st) {
  accept_kernel<<<dim3(a.B), dim3(LLMCAD_MAX_NODES), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace llmcad
