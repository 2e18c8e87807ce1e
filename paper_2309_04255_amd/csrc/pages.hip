// Pages of requests between steps: requests that continue from others' tokens (fork),
// and the pages in use moved to the front of the pool (compact).
//
// Every workgroup decides for itself: it marks the pages that the requests hold in a bitmap
// in LDS (a few KiB of table entries, read by all), counts the free ones, and knows then
// which page goes where; it writes its share of the new tables and lists and copies its
// share of the pages.  Nothing is handed from one workgroup to another, so one launch is
// enough.  Pools of more than 256 requests or 2^16 pages, long tables, and forks of many
// heads, take two, one that decides and leaves the copies in the workspace, and one that
// copies.
//
// Bound by bytes where pages are whole: a 7B pool's 34 moves (1.14 GB each way) take 453 to 459 us
// (4970 to 5040 GB/s).  A fork copies parts of pages, and of V^T parts of lines, which memory reads
// and writes whole: 19 copies of 32 tokens on average of 40 layers of 8 heads, 99 MB, are
// 229 MB read and 125 written (copies 81 us, deciding 10).  Small ones are a chain of
// latencies: lengths, tables, two counts, the copies (four requests of the ~1B model 12 us, a
// pool of 300 pages of 64 KiB 9.7).
#include "batch.h"

namespace llmcad {

namespace {

constexpr int kGroup = 8;     // bitmap words per thread
constexpr int kSmall = 256;   // threads of the one launch: its most requests, 256 of its pages each
constexpr int kLarge = 1024;
static_assert(LLMCAD_MAX_POOL <= kLarge * kGroup * 32 && kMaxRequests <= kLarge, "every request and bitmap word has a thread");

// Sum of v over the threads before this one; `total` over all.  Called by all threads.
template <int THREADS>
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
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) {
    if (w < wave) before += lds[w];
    total += lds[w];
  }
  return before + sum - v;
}

template <int THREADS>
struct Bitmap {
  uint32_t word[THREADS * kGroup];
  int zeros[THREADS];  // clear bits before each group of words

  __device__ __forceinline__ void clear(int n) {
    for (int e = threadIdx.x; e < (n + 31) / 32; e += THREADS) word[e] = 0;
  }
  __device__ __forceinline__ void set(int p) { atomicOr(&word[p >> 5], 1u << (p & 31)); }
  __device__ __forceinline__ bool has(int p) const { return word[p >> 5] >> (p & 31) & 1; }
  // The clear (or set) bits of word w among the first n pages.
  template <bool SET>
  __device__ __forceinline__ uint32_t bits(int w, int n) const {
    const int left = n - 32 * w;
    return left <= 0 ? 0u : (SET ? word[w] : ~word[w]) & (left >= 32 ? ~0u : (1u << left) - 1);
  }
  // Counts the clear bits of the first n pages; called by all threads, after the marks.
  __device__ __forceinline__ int count(int n, int* lds) {
    int mine = 0, total;
    const int w0 = threadIdx.x * kGroup;
    for (int w = w0; w < w0 + kGroup && 32 * w < n; ++w) mine += __popc(bits<false>(w, n));
    zeros[threadIdx.x] = block_before<THREADS>(mine, lds, total);
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
  // The k-th clear (or set) bit of the first n pages (there are more than k).
  template <bool SET>
  __device__ __forceinline__ int nth(int k, int n) const {
    const auto before = [&](int g) { return SET ? g * kGroup * 32 - zeros[g] : zeros[g]; };
    int lo = 0, hi = ((n + 31) / 32 + kGroup - 1) / kGroup - 1;  // the last group with at most k before it
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (before(mid) <= k) lo = mid;
      else hi = mid - 1;
    }
    k -= before(lo);
    for (int w = lo * kGroup; 32 * w < n; ++w) {
      uint32_t b = bits<SET>(w, n);
      const int c = __popc(b);
      if (k < c) {
        for (; k > 0; --k) b &= b - 1;
        return 32 * w + __ffs(b) - 1;
      }
      k -= c;
    }
    return 0;
  }
};

__device__ __forceinline__ int pages_of(int held) { return (int)(((long long)held + kPage - 1) / kPage); }

// f(request, page) for every page that the lengths in LDS say is held; `widest` is
// the most pages of a request.  (At most 2^10 tables of 2^18 columns.)
template <int THREADS, class F>
__device__ __forceinline__ void each_page(const PagesArgs& a, const int* held, int widest, F f) {
  if (widest == 0) return;
  constexpr int AHEAD = 4;  // loads in flight
  const int rows = THREADS / widest, cols = THREADS % widest;  // (a step of the loop, without a division)
  int b = threadIdx.x / widest, col = threadIdx.x % widest;
  while (b < a.B) {
    int page[AHEAD], of[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      page[i] = -1;
      of[i] = b;
      if (b < a.B && col < pages_of(held[b])) page[i] = ldg(a.table + (size_t)b * a.max_pages + col);
      b += rows;
      col += cols;
      if (col >= widest) {
        col -= widest;
        ++b;
      }
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (page[i] >= 0 && page[i] < a.n_pages) f(of[i], page[i]);
  }
}

template <int THREADS>
struct Fork {
  Bitmap<THREADS> before, after;
  int held[THREADS], source[THREADS], first[THREADS];
  int page[THREADS];  // the page of a request's copied last tokens, -1: none
  uint8_t alive[THREADS];
  int lds[THREADS / kWave], widest;
  PageCopy copies[THREADS];

  // Returns the number of copies; called by all threads of every workgroup, of which the first
  // G write the new tables and lists.
  __device__ __forceinline__ int decide(const PagesArgs& a, int G) {
    const int tid = threadIdx.x, B = a.B, g = blockIdx.x;
    int mine = 0, from = -1;
    bool bad = false;
    if (tid < B) {
      mine = ldg(a.held + tid);
      from = ldg(a.source + tid);
      bad = mine < 0 || pages_of(mine) > a.max_pages || from >= B;
      held[tid] = mine;
      source[tid] = from;
      first[tid] = B;
      alive[tid] = 0;
      page[tid] = -1;
    }
    before.clear(a.n_pages);
    after.clear(a.n_pages);
    if (tid == 0) widest = 0;
    int status = __syncthreads_or(bad) ? LLMCAD_PLAN_BAD_LENGTHS : LLMCAD_PLAN_OK, n_copies = 0;
    if (status == LLMCAD_PLAN_OK) {
      if (tid < B) {
        atomicMax(&widest, pages_of(mine));
        if (from >= 0) {
          alive[from] = 1;
          atomicMin(&first[from], tid);
        }
      }
      __syncthreads();
      // who needs a page of its own for its last tokens
      PageCopy c{};
      bool copies_one = false;
      if (tid < B && from >= 0 && from != tid) {
        c.rows = held[from] % kPage;
        copies_one = c.rows > 0 && !(source[from] != from && first[from] == tid);  // (the first of a source that moved goes on with it)
        if (copies_one) c.src = ldg(a.table + (size_t)from * a.max_pages + held[from] / kPage);
      }
      // the pages held before, and those that somebody still holds
      each_page<THREADS>(a, held, widest, [&](int b, int p) {
        before.set(p);
        if (alive[b]) after.set(p);
      });
      if (copies_one) copies_one = c.src >= 0 && c.src < a.n_pages;
      __syncthreads();
      const int n_free = before.count(a.n_pages, lds), k = block_before<THREADS>(copies_one ? 1 : 0, lds, n_copies);
      if (n_copies > n_free) {
        status = LLMCAD_PLAN_NO_PAGES;
        n_copies = 0;
      } else if (copies_one) {
        c.dst = before.template nth<false>(k, a.n_pages);
        page[tid] = c.dst;
        after.set(c.dst);
        copies[k] = c;
      }
    }
    __syncthreads();
    const bool ok = status == LLMCAD_PLAN_OK;
    if (g >= G) return n_copies;
    const int left = ok ? after.count(a.n_pages, lds) : 0;  // (pages nobody holds now)
    // tables and lengths: a workgroup's share
    for (int e = g * THREADS + tid; e < B * a.max_pages; e += G * THREADS) {
      const int b = e / a.max_pages, col = e % a.max_pages, s = ok ? source[b] : b;
      const int have = ok ? (s < 0 ? 0 : pages_of(held[s])) : a.max_pages;
      int p = -1;
      if (col < have) p = ldg(a.table + (size_t)s * a.max_pages + col);
      if (ok && page[b] >= 0 && col == have - 1) p = page[b];
      stg(a.table_out + e, p);
    }
    // the free list: pages in order, then -1
    if (ok)
      for (int p = g * THREADS + tid; p < a.n_pages; p += G * THREADS)
        if (!after.has(p)) stg(a.free_pages + after.zeros_before(p), p);
    for (int i = left + g * THREADS + tid; i < a.n_pages; i += G * THREADS) stg(a.free_pages + i, -1);
    if (g == 0) {
      if (tid < B) stg(a.held_out + tid, !ok ? mine : from < 0 ? 0 : held[from]);
      if (tid == 0) {
        stg(a.n_free, left);
        stg(a.status, status);
      }
    }
    return n_copies;
  }
};

template <int THREADS>
struct Compact {
  Bitmap<THREADS> used;
  int held[THREADS];
  int lds[THREADS / kWave], widest;
  int n_used;

  __device__ __forceinline__ int decide(const PagesArgs& a) {
    const int tid = threadIdx.x, B = a.B, g = blockIdx.x, G = gridDim.x;
    int mine = 0;
    if (tid < B) {
      mine = ldg(a.held + tid);
      if (mine < 0) mine = 0;
      if (pages_of(mine) > a.max_pages) mine = (int)((long long)a.max_pages * kPage);
      held[tid] = mine;
    }
    used.clear(a.n_pages);
    if (tid == 0) widest = 0;
    __syncthreads();
    if (tid < B) atomicMax(&widest, pages_of(mine));
    __syncthreads();
    each_page<THREADS>(a, held, widest, [&](int, int p) { used.set(p); });
    __syncthreads();
    const int in_use = a.n_pages - used.count(a.n_pages, lds);
    const int n = in_use < a.n_pages ? used.zeros_before(in_use) : 0;  // free pages in front of the new end
    for (int e = g * THREADS + tid; e < B * a.max_pages; e += G * THREADS) {
      const int b = e / a.max_pages, col = e % a.max_pages;
      int p = -1;
      if (col < pages_of(held[b])) {
        p = ldg(a.table + e);
        if (p < 0 || p >= a.n_pages) p = -1;
        else if (p >= in_use) p = used.template nth<false>((p - in_use) - (used.zeros_before(p) - n), a.n_pages);
      }
      stg(a.table_out + e, p);
    }
    if (g == 0 && tid == 0) stg(a.n_used, in_use);
    n_used = in_use;
    return n;
  }
  // The k-th used page behind the end takes the k-th of the n free ones before it.
  __device__ __forceinline__ PageCopy copy(const PagesArgs& a, int k, int n) const {
    return {used.template nth<true>(n_used - n + k, a.n_pages), used.template nth<false>(k, a.n_pages), kPage};
  }
};

constexpr int kWriters = 32;

// ---------------------------------------------------------------- copies
constexpr int kCopyThreads = 256;

// A head's first `rows` keys (one run of memory) and the first `rows` entries of each
// dim's line of values, in 16-byte pieces, all loads before the first store.  Lines are
// written in whole pieces of kWhole entries, in which what lies behind the copied ones is
// read from the new page first: memory takes smaller parts by reading them itself, later
// (32 copies of 320 heads with 63 tokens 187 us for 219 entry by entry, 33 tokens 156 for 182;
// with 1 to 16 tokens 7 to 10% slower; whole lines instead of halves: the same above 32, 154 for 122 at 32).
constexpr int kWhole = 32;
template <int DH>
__device__ __forceinline__ void copy_head(const bf16x8* ks, bf16x8* kd, const bf16x8* vs, bf16x8* vd, int rows) {
  constexpr int PER = kPage * DH / 8 / kCopyThreads;
  const int n = rows * (DH / 8);                                            // pieces of the keys
  const int line = (rows + kWhole - 1) / kWhole * (kWhole / 8), m = DH * line;  // of a line of values, and of all
  bf16x8 k[PER], v[PER], old[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = threadIdx.x + i * kCopyThreads;
    if (e < n) k[i] = ldg(ks + e);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = threadIdx.x + i * kCopyThreads;
    if (e >= m) continue;
    const int at = e / line * 8 + e % line, left = rows - 8 * (e % line);
    if (left > 0) v[i] = ldg(vs + at);
    if (left < 8) old[i] = ldg(vd + at);
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
    const int left = rows - 8 * (e % line);
    bf16x8 x = v[i];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bf16 mine = v[i][u], there = old[i][u];
      x[u] = u < left ? mine : there;
    }
    stg(vd + e / line * 8 + e % line, x);
  }
}

// This workgroup's share of n copies' page heads: copy_of(k) is the k-th.
template <int DH, class F>
__device__ __forceinline__ void copy_units(const PagesArgs& a, int n, F copy_of) {
  const int heads = a.L * a.Hkv;
  const size_t head = (size_t)kPage * DH / 8;  // (in pieces)
  int k = -1;
  PageCopy c{};
  for (long long unit = blockIdx.x; unit < (long long)n * heads; unit += gridDim.x) {
    const int at = (int)(unit % heads), layer = at / a.Hkv, kh = at % a.Hkv;
    if ((int)(unit / heads) != k) {
      k = (int)(unit / heads);
      c = copy_of(k);
    }
    const size_t src = (((size_t)layer * a.n_pages + c.src) * a.Hkv + kh) * head;
    const size_t dst = (((size_t)layer * a.n_pages + c.dst) * a.Hkv + kh) * head;
    copy_head<DH>((const bf16x8*)a.k_pages + src, (bf16x8*)a.k_pages + dst, (const bf16x8*)a.v_pages + src,
                  (bf16x8*)a.v_pages + dst, c.rows);
  }
}
template <int DH>
__global__ __launch_bounds__(kSmall) void fork_kernel(PagesArgs a) {
  __shared__ Fork<kSmall> f;
  const int n = f.decide(a, min(kWriters, (int)gridDim.x));
  copy_units<DH>(a, n, [&](int k) { return f.copies[k]; });
}
template <int DH>
__global__ __launch_bounds__(kSmall) void compact_kernel(PagesArgs a) {
  __shared__ Compact<kSmall> f;
  const int n = f.decide(a);
  __syncthreads();
  copy_units<DH>(a, n, [&](int k) { return f.copy(a, k, n); });
}

__global__ __launch_bounds__(kLarge) void fork_plan_kernel(PagesArgs a) {
  __shared__ Fork<kLarge> f;
  const int n = f.decide(a, gridDim.x), k = threadIdx.x;
  if (blockIdx.x != 0) return;
  if (k < n) stg(a.copies + k, f.copies[k]);
  if (k == 0) stg(a.n_copies, n);
}
__global__ __launch_bounds__(kLarge) void compact_plan_kernel(PagesArgs a) {
  __shared__ Compact<kLarge> f;
  const int n = f.decide(a);
  __syncthreads();
  for (int k = blockIdx.x * kLarge + threadIdx.x; k < n; k += gridDim.x * kLarge) stg(a.copies + k, f.copy(a, k, n));
  if (blockIdx.x == 0 && threadIdx.x == 0) stg(a.n_copies, n);
}
template <int DH>
__global__ __launch_bounds__(kCopyThreads) void copy_kernel(PagesArgs a) {
  const int n = ldg(a.n_copies);
  copy_units<DH>(a, n, [&](int k) { return ldg(a.copies + k); });
}

// Workgroups that copy: six on a CU, no more than there are heads of `most` copies.
int copy_groups(const PagesArgs& a, long long most) {
  const long long units = most * a.L * a.Hkv;
  return (int)(units < 1 ? 1 : units > 1536 ? 1536 : units);
}
// Workgroups that share the writes of a large plan: one per 4096 pages or table entries.
int plan_groups(const PagesArgs& a) {
  const long long n = ((long long)a.B * a.max_pages + a.n_pages) / 4096;
  return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}
// (Every workgroup of the one launch reads all tables, up to so many entries.)
bool is_small(const PagesArgs& a, int most_entries) {
  return a.B <= kSmall && a.n_pages <= kSmall * kGroup * 32 && (long long)a.B * a.max_pages <= most_entries;
}

void launch_copies(const PagesArgs& a, long long most, hipStream_t st) {
  if (a.Dh == 128)
    copy_kernel<128><<<dim3(copy_groups(a, most)), dim3(kCopyThreads), 0, st>>>(a);
  else
    copy_kernel<64><<<dim3(copy_groups(a, most)), dim3(kCopyThreads), 0, st>>>(a);
}

}  // namespace

hipError_t launch_batch_fork(const PagesArgs& a, hipStream_t st) {
  // (One launch: four requests of 22 layers of 16 heads 11.9 us for 14.6 with two; 64 of 40 layers of 8 heads, where
  // the deciding part's registers and LDS cost the copies' waves, 99 for 93.  The limits lie between these sizes,
  // none of which between was timed; the copies may be few, which the device alone knows.)
  if (!is_small(a, 2048) || (long long)a.B * a.L * a.Hkv > 4096) {
    fork_plan_kernel<<<dim3(plan_groups(a)), dim3(kLarge), 0, st>>>(a);
    launch_copies(a, a.B, st);
  } else if (a.Dh == 128) {
    fork_kernel<128><<<dim3(copy_groups(a, a.B)), dim3(kSmall), 0, st>>>(a);
  } else {
    fork_kernel<64><<<dim3(copy_groups(a, a.B)), dim3(kSmall), 0, st>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_batch_compact(const PagesArgs& a, hipStream_t st) {
  // (2300 entries: 13.2 us, with two launches 14.5; the fork of 193 requests of 24 columns 30 for 23.)
  if (!is_small(a, 8192)) {
    compact_plan_kernel<<<dim3(plan_groups(a)), dim3(kLarge), 0, st>>>(a);
    launch_copies(a, a.n_pages / 2, st);
  } else if (a.Dh == 128) {
    compact_kernel<128><<<dim3(copy_groups(a, a.n_pages / 2)), dim3(kSmall), 0, st>>>(a);
  } else {
    compact_kernel<64><<<dim3(copy_groups(a, a.n_pages / 2)), dim3(kSmall), 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace llmcad
