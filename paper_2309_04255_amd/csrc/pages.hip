// Pages of requests between steps: requests that continue from others' tokens (fork),
// and the pages in use moved to the front of the pool (compact).
//
// Both begin with one small launch that decides: every workgroup marks the pages that
// the requests hold in a bitmap in LDS (a few KiB of table entries, read by all), counts
// the free ones, and writes its share of the new tables and lists; nothing is handed from
// one workgroup to another.  A second launch copies, as many workgroups as fill the GPU
// striding over (copy, layer, K/V head).
#include "batch.h"

namespace llmcad {

namespace {

constexpr int kThreads = 1024;
constexpr int kGroup = 8;  // bitmap words per thread
constexpr int kMaxPool = LLMCAD_MAX_POOL;
static_assert(kMaxPool <= kThreads * kGroup * 32, "a bitmap word of every page has a thread");
static_assert(kMaxRequests <= kThreads, "a request has a thread");

// Sum of v over the threads before this one; `total` over all.  Called by all threads.
__device__ __forceinline__ int block_before(int v, int* lds, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int sum = v;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int o = __shfl_up(sum, off, kWave);
    if (lane >= off) sum += o;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = sum;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int w = 0; w < kThreads / kWave; ++w) {
    if (w < wave) before += lds[w];
    total += lds[w];
  }
  return before + sum - v;
}

struct Bitmap {
  uint32_t word[kMaxPool / 32];
  int zeros[kThreads];  // clear bits before each group of words

  __device__ __forceinline__ void clear(int n) {
    for (int e = threadIdx.x; e < (n + 31) / 32; e += kThreads) word[e] = 0;
  }
  __device__ __forceinline__ void set(int p) { atomicOr(&word[p >> 5], 1u << (p & 31)); }
  __device__ __forceinline__ bool has(int p) const { return word[p >> 5] >> (p & 31) & 1; }
  // The clear bits of word w among the first n pages.
  __device__ __forceinline__ uint32_t clear_bits(int w, int n) const {
    const int left = n - 32 * w;
    return left <= 0 ? 0u : ~word[w] & (left >= 32 ? ~0u : (1u << left) - 1);
  }
  // Counts the clear bits of the first n pages; called by all threads, after the marks.
  __device__ __forceinline__ int count(int n, int* lds) {
    int mine = 0, total;
    const int w0 = threadIdx.x * kGroup;
    for (int w = w0; w < w0 + kGroup && 32 * w < n; ++w) mine += __popc(clear_bits(w, n));
    const int before = block_before(mine, lds, total);
    zeros[threadIdx.x] = before;
    __syncthreads();
    return total;
  }
  // Clear bits before page p (after count).
  __device__ __forceinline__ int zeros_before(int p) const {
    const int w = p >> 5, g = w / kGroup;
    int z = zeros[g];
    for (int i = g * kGroup; i < w; ++i) z += __popc(~word[i]);
    return z + __popc(~word[w] & ((1u << (p & 31)) - 1));
  }
  // The k-th clear bit of the first n pages (there are more than k).
  __device__ __forceinline__ int nth_zero(int k, int n) const {
    const int groups = ((n + 31) / 32 + kGroup - 1) / kGroup;
    int lo = 0, hi = groups - 1;  // the last group with zeros[g] <= k
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (zeros[mid] <= k) lo = mid;
      else hi = mid - 1;
    }
    k -= zeros[lo];
    for (int w = lo * kGroup; 32 * w < n; ++w) {
      uint32_t bits = clear_bits(w, n);
      const int c = __popc(bits);
      if (k < c) {
        for (; k > 0; --k) bits &= bits - 1;
        return 32 * w + __ffs(bits) - 1;
      }
      k -= c;
    }
    return 0;
  }
};

__device__ __forceinline__ int pages_of(int held) { return (int)(((long long)held + kPage - 1) / kPage); }

__global__ __launch_bounds__(kThreads) void fork_plan_kernel(PagesArgs a) {
  __shared__ Bitmap before, after;
  __shared__ int held_s[kMaxRequests], source_s[kMaxRequests], first_s[kMaxRequests];
  __shared__ int page_s[kMaxRequests];  // the page of a request's copied last tokens, -1: none
  __shared__ uint8_t alive_s[kMaxRequests];
  __shared__ int lds[kThreads / kWave], widest_s;
  const int tid = threadIdx.x, B = a.B, g = blockIdx.x, G = gridDim.x;
  before.clear(a.n_pages);
  after.clear(a.n_pages);
  int held = 0, source = -1;
  bool bad = false;
  if (tid < B) {
    held = ldg(a.held + tid);
    source = ldg(a.source + tid);
    bad = held < 0 || pages_of(held) > a.max_pages || source >= B;
    held_s[tid] = held;
    source_s[tid] = source;
    first_s[tid] = B;
    alive_s[tid] = 0;
    page_s[tid] = -1;
  }
  if (tid == 0) widest_s = 0;
  bad = __syncthreads_or(bad) != 0;
  int status = bad ? LLMCAD_PLAN_BAD_LENGTHS : LLMCAD_PLAN_OK;
  if (!bad) {
    if (tid < B) {
      atomicMax(&widest_s, pages_of(held));
      if (source >= 0) {
        alive_s[source] = 1;
        atomicMin(&first_s[source], tid);
      }
    }
    __syncthreads();
    // the pages held before, and those that somebody still holds
    const int widest = widest_s, entries = B * widest;  // (at most 2^10 tables of 2^18 pages)
#pragma unroll 4
    for (int e = tid; e < entries; e += kThreads) {
      const int b = e / widest, col = e % widest;
      if (col < pages_of(held_s[b])) {
        const int p = ldg(a.table + (size_t)b * a.max_pages + col);
        if (p >= 0 && p < a.n_pages) {
          before.set(p);
          if (alive_s[b]) after.set(p);
        }
      }
    }
    __syncthreads();
    const int n_free = before.count(a.n_pages, lds);
    // who needs a page of its own for its last tokens
    PageCopy c{};
    bool copies = false;
    if (tid < B && source >= 0 && source != tid) {
      const int from = held_s[source], col = from / kPage;
      c.rows = from % kPage;
      const bool goes_on = source_s[source] != source && first_s[source] == tid;
      if (c.rows > 0 && !goes_on) {
        c.src = ldg(a.table + (size_t)source * a.max_pages + col);
        copies = c.src >= 0 && c.src < a.n_pages;
      }
    }
    int n_copies;
    const int k = block_before(copies ? 1 : 0, lds, n_copies);
    if (n_copies > n_free) {
      status = LLMCAD_PLAN_NO_PAGES;
    } else {
      if (copies) {
        c.dst = before.nth_zero(k, a.n_pages);
        page_s[tid] = c.dst;
        after.set(c.dst);
        if (g == 0) stg(a.copies + k, c);
      }
      if (g == 0 && tid == 0) stg(a.n_copies, n_copies);
    }
  }
  __syncthreads();
  const bool ok = status == LLMCAD_PLAN_OK;
  const int left = ok ? after.count(a.n_pages, lds) : 0;  // (pages nobody holds now)
  // tables and lengths: a workgroup's share
#pragma unroll 4
  for (int e = g * kThreads + tid; e < B * a.max_pages; e += G * kThreads) {
    const int b = e / a.max_pages, col = e % a.max_pages, s = ok ? source_s[b] : b;
    const int have = ok ? (s < 0 ? 0 : pages_of(held_s[s])) : a.max_pages;
    int p = -1;
    if (col < have) p = ldg(a.table + (size_t)s * a.max_pages + col);
    if (ok && page_s[b] >= 0 && col == have - 1) p = page_s[b];
    stg(a.table_out + e, p);
  }
  if (g == 0 && tid < B) stg(a.held_out + tid, !ok ? held : source < 0 ? 0 : held_s[source]);
  // the free list: pages in order, then -1
  if (ok) {
    const int pairs = (a.n_pages + 63) / 64, wave = g * (kThreads / kWave) + (tid >> 6), lane = tid & 63;
    for (int w = wave; w < pairs; w += G * (kThreads / kWave)) {
      const int p = 64 * w + lane;
      if (p < a.n_pages && !after.has(p)) stg(a.free_pages + after.zeros_before(p), p);
    }
  }
  for (int i = left + g * kThreads + tid; i < a.n_pages; i += G * kThreads) stg(a.free_pages + i, -1);
  if (g == 0 && tid == 0) {
    stg(a.n_free, left);
    stg(a.status, status);
    if (!ok) stg(a.n_copies, 0);
  }
}

__global__ __launch_bounds__(kThreads) void compact_plan_kernel(PagesArgs a) {
  __shared__ Bitmap used;
  __shared__ int held_s[kMaxRequests];
  __shared__ int lds[kThreads / kWave], widest_s;
  const int tid = threadIdx.x, B = a.B, g = blockIdx.x, G = gridDim.x;
  used.clear(a.n_pages);
  if (tid == 0) widest_s = 0;
  __syncthreads();
  if (tid < B) {
    int held = ldg(a.held + tid);
    if (held < 0) held = 0;
    if (pages_of(held) > a.max_pages) held = (int)((long long)a.max_pages * kPage);
    held_s[tid] = held;
    atomicMax(&widest_s, pages_of(held));
  }
  __syncthreads();
  const int widest = widest_s, entries = B * widest;
#pragma unroll 4
  for (int e = tid; e < entries; e += kThreads) {
    const int b = e / widest, col = e % widest;
    if (col < pages_of(held_s[b])) {
      const int p = ldg(a.table + (size_t)b * a.max_pages + col);
      if (p >= 0 && p < a.n_pages) used.set(p);
    }
  }
  __syncthreads();
  const int n_used = a.n_pages - used.count(a.n_pages, lds);
  const int moves = n_used < a.n_pages ? used.zeros_before(n_used) : 0;  // free pages in front of the new end
  // The k-th used page behind the end takes the k-th free one before it.
  const int pairs = (a.n_pages + 63) / 64, wave = g * (kThreads / kWave) + (tid >> 6), lane = tid & 63;
  for (int w = wave; w < pairs; w += G * (kThreads / kWave)) {
    const int p = 64 * w + lane;
    if (p >= a.n_pages) continue;
    if (p < n_used && !used.has(p)) stg(&a.copies[used.zeros_before(p)].dst, p);
    if (p >= n_used && used.has(p)) {
      PageCopy* c = a.copies + (p - n_used) - (used.zeros_before(p) - moves);
      stg(&c->src, p);
      stg(&c->rows, kPage);
    }
  }
  for (int e = g * kThreads + tid; e < B * a.max_pages; e += G * kThreads) {
    const int b = e / a.max_pages, col = e % a.max_pages;
    int p = -1;
    if (col < pages_of(held_s[b])) {
      p = ldg(a.table + e);
      if (p < 0 || p >= a.n_pages) p = -1;
      else if (p >= n_used) p = used.nth_zero((p - n_used) - (used.zeros_before(p) - moves), a.n_pages);
    }
    stg(a.table_out + e, p);
  }
  if (g == 0 && tid == 0) {
    stg(a.n_used, n_used);
    stg(a.n_copies, moves);
  }
}

// ---------------------------------------------------------------- copies
constexpr int kCopyThreads = 256;

// A head's first `rows` keys (one run of memory) and the first `rows` entries of each
// dim's line of values, in 16-byte pieces, all loads before the first store.  The piece
// of a line that they end in is written entry by entry, so that what lies behind stays.
template <int DH>
__device__ __forceinline__ void copy_head(const bf16x8* ks, bf16x8* kd, const bf16x8* vs, bf16x8* vd, int rows) {
  constexpr int PER = kPage * DH / 8 / kCopyThreads;
  const int n = rows * (DH / 8), line = (rows + 7) / 8, m = DH * line;  // pieces of the keys, of a line, of the values
  bf16x8 k[PER], v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = threadIdx.x + i * kCopyThreads;
    if (e < n) k[i] = ldg(ks + e);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = threadIdx.x + i * kCopyThreads;
    if (e < m) v[i] = ldg(vs + e / line * 8 + e % line);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = threadIdx.x + i * kCopyThreads;
    if (e < n) stg(kd + e, k[i]);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = threadIdx.x + i * kCopyThreads;
    if (e >= m) continue;
    bf16x8* to = vd + e / line * 8 + e % line;
    const int left = rows - 8 * (e % line);
    if (left >= 8) {
      stg(to, v[i]);
    } else {
#pragma unroll
      for (int u = 0; u < 7; ++u) {
        const bf16 x = v[i][u];
        if (u < left) stg((bf16*)to + u, x);
      }
    }
  }
}

template <int DH>
__global__ __launch_bounds__(kCopyThreads) void copy_kernel(PagesArgs a) {
  const int n = ldg(a.n_copies), heads = a.L * a.Hkv;
  const size_t head = (size_t)kPage * DH / 8;  // (in pieces)
  for (long long unit = blockIdx.x; unit < (long long)n * heads; unit += gridDim.x) {
    const PageCopy c = ldg(a.copies + unit / heads);
    const int at = (int)(unit % heads), layer = at / a.Hkv, kh = at % a.Hkv;
    const size_t src = (((size_t)layer * a.n_pages + c.src) * a.Hkv + kh) * head;
    const size_t dst = (((size_t)layer * a.n_pages + c.dst) * a.Hkv + kh) * head;
    copy_head<DH>((const bf16x8*)a.k_pages + src, (bf16x8*)a.k_pages + dst, (const bf16x8*)a.v_pages + src,
                  (bf16x8*)a.v_pages + dst, c.rows);
  }
}

hipError_t launch_copies(const PagesArgs& a, long long most, hipStream_t st) {
  const long long units = most * a.L * a.Hkv;
  const dim3 grid((unsigned)(units < 2048 ? (units < 1 ? 1 : units) : 2048));
  if (a.Dh == 128)
    copy_kernel<128><<<grid, dim3(kCopyThreads), 0, st>>>(a);
  else
    copy_kernel<64><<<grid, dim3(kCopyThreads), 0, st>>>(a);
  return hipGetLastError();
}

// Workgroups that share the writes of a plan: one per 4096 pages or table entries.
int plan_groups(const PagesArgs& a) {
  const long long writes = (long long)a.B * a.max_pages + a.n_pages, n = writes / 4096;
  return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}

}  // namespace

hipError_t launch_batch_fork(const PagesArgs& a, hipStream_t st) {
  fork_plan_kernel<<<dim3(plan_groups(a)), dim3(kThreads), 0, st>>>(a);
  return launch_copies(a, a.B, st);
}

hipError_t launch_batch_compact(const PagesArgs& a, hipStream_t st) {
  compact_plan_kernel<<<dim3(plan_groups(a)), dim3(kThreads), 0, st>>>(a);
  return launch_copies(a, a.n_pages / 2, st);
}

}  // namespace llmcad
