// A step of several requests behind one shared prefix, around its attention:
// the plan (pages, slots, positions, ancestor masks, rotary table), the rotary
// embedding with the write of the new keys and values into pages, and the
// rollback to the accepted rows.
#include "batch.h"

namespace llmcad {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int up_div(int x, int a) { return (x + a - 1) / a; }

// Sum of a pair of 64-bit values over the workgroup, in every thread.
__device__ __forceinline__ void block_sum(long long (&v)[4], long long* lds) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v[i] += __shfl_xor(v[i], off, kWave);
  __syncthreads();
  if ((threadIdx.x & 63) == 0)
    for (int i = 0; i < 4; ++i) lds[(threadIdx.x >> 6) * 4 + i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = 0;
    for (int w = 0; w < kThreads / kWave; ++w) v[i] += lds[w * 4 + i];
  }
  __syncthreads();
}

// One workgroup per request.  Every workgroup reads all requests' lengths (a
// few KiB) and sums what lies before its own, so that nothing is handed from
// one workgroup to another and the launch needs no counters.  Ancestors by pointer
// jumping: after round i a row's mask holds its 2^i nearest and `up` the next one.
// Bound by the chain of its steps (lengths, two sums, pages, parents, seven rounds,
// sines), each a latency: 8.2 us for one request of 31 rows, 10.3 us for 256 of up
// to 41 (2.9 MB written; 0.6 us of a copy).
__global__ __launch_bounds__(kThreads) void plan_kernel(PlanArgs a) {
  __shared__ long long sums[4 * kThreads / kWave];
  __shared__ int up[128];
  __shared__ uint32_t anc[128][4];
  __shared__ int pos_s[128];
  __shared__ int page_s[4];
  __shared__ int bad_s;
  const int b = blockIdx.x, tid = threadIdx.x, B = a.B;
  constexpr int PER = kMaxRequests / kThreads;
  int n[PER], held[PER];
  int bad = 0;
  // pages wanted before request b and in all, pages held in all, (row, page) pairs in all
  long long v[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = tid + i * kThreads;
    n[i] = held[i] = 0;
    if (r < B) {
      const int lo = ldg(a.row_start + r), hi = ldg(a.row_start + r + 1);
      const int h = ldg(a.held + r);
      if (lo < 0 || hi < lo || (long long)hi - lo > LLMCAD_MAX_NODES || hi > a.N || h < 0 || (r == 0 && lo != 0)) {
        bad = 1;
      } else {
        n[i] = hi - lo;
        held[i] = h;
      }
      const long long need = ((long long)held[i] + n[i] + kPage - 1) / kPage - ((long long)held[i] + kPage - 1) / kPage;
      long long pages = ((long long)held[i] + n[i] + kPage - 1) / kPage;
      if (pages > a.max_pages) pages = a.max_pages;
      if (r < b) v[0] += need;
      v[1] += need;
      if (n[i] > 0) v[2] += pages;
      v[3] += pages * n[i];
    }
  }
  const bool invalid = __syncthreads_or(bad) != 0;
  block_sum(v, sums);
  const long long need_before = v[0];
  // The length of a run of pages: see kSplitRuns and kSplitRows; at least two
  // pages, 32 keys for each of a workgroup's four waves.
  long long chunk = 2;
  const long long c1 = (v[2] + kSplitRuns - 1) / kSplitRuns;
  const long long room = a.N > kSplitRows ? a.N : kSplitRows;
  const long long c2 = (v[3] + room - 1) / room;
  if (c1 > chunk) chunk = c1;
  if (c2 > chunk) chunk = c2;
  const long long taken = v[1];
  // runs before request b and in all, partial rows before it
  long long w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = tid + i * kThreads;
    if (r < B && n[i] > 0) {
      long long pages = ((long long)held[i] + n[i] + kPage - 1) / kPage;
      if (pages > a.max_pages) pages = a.max_pages;
      const long long ns = (pages + chunk - 1) / chunk;
      if (r < b) {
        w[0] += ns;
        w[2] += ns * n[i];
      }
      w[1] += ns;
    }
  }
  block_sum(w, sums);
  const int row0 = invalid ? 0 : ldg(a.row_start + b);
  const int nb = invalid ? 0 : ldg(a.row_start + b + 1) - row0;
  const int hb = invalid ? 0 : ldg(a.held + b);
  const long long end = (long long)hb + nb;
  const int first_new = (int)(((long long)hb + kPage - 1) / kPage);
  const int need = (int)((end + kPage - 1) / kPage) - first_new;
  int ns = 0;
  if (nb > 0) {
    long long pages = (end + kPage - 1) / kPage;
    if (pages > a.max_pages) pages = a.max_pages;
    ns = (int)((pages + chunk - 1) / chunk);
  }

  // Pages: the one the first new row shares with held tokens, then free ones.
  if (tid == 0) bad_s = 0;
  __syncthreads();
  int st = LLMCAD_PLAN_OK;
  if (invalid) st = LLMCAD_PLAN_BAD_LENGTHS;
  else if (nb > 0 && (end > (long long)a.max_pages * kPage || need_before + need > a.n_free || a.prefix_len + end > 1ll << 31))
    st = LLMCAD_PLAN_NO_PAGES;  // (the last: a position that is no int32)
  const int col0 = hb / kPage;  // table column of the first new row
  if (st == LLMCAD_PLAN_OK && nb > 0 && tid < 4) {
    const int col = col0 + tid;
    int id = -1;
    if ((long long)col * kPage < end) {
      id = col < first_new ? ldg(a.table + (size_t)b * a.max_pages + col)
                           : ldg(a.free_pages + need_before + (col - first_new));
      if (id < 0 || id >= a.n_pages) bad_s = 1;
    }
    page_s[tid] = id;
  }
  __syncthreads();
  if (st == LLMCAD_PLAN_OK && bad_s) st = LLMCAD_PLAN_NO_PAGES;

  // Parents, then ancestors-or-self by pointer jumping (7 rounds cover 128 rows).
  int parent = -1;
  bad = 0;
  if (st == LLMCAD_PLAN_OK && tid < nb) {
    parent = a.parent ? ldg(a.parent + row0 + tid) : tid - 1;
    if (tid == 0 ? parent != -1 : (parent < 0 || parent >= tid)) bad = 1;
  }
  if (__syncthreads_or(bad)) st = LLMCAD_PLAN_BAD_TREE;
  const bool placed = st == LLMCAD_PLAN_OK;
  if (placed && tid < 4 && nb > 0) {
    const int col = col0 + tid;
    if (col >= first_new && (long long)col * kPage < end) stg(a.table + (size_t)b * a.max_pages + col, page_s[tid]);
  }
  if (placed && tid < nb) {
    up[tid] = parent;
#pragma unroll
    for (int j = 0; j < 4; ++j) anc[tid][j] = (tid >> 5) == j ? 1u << (tid & 31) : 0u;
  }
  __syncthreads();
  for (int round = 0; round < 7; ++round) {
    uint32_t m[4] = {0, 0, 0, 0};
    int next = -1;
    const bool on = placed && tid < nb && up[tid] >= 0;
    if (on) {
      const int p = up[tid];
      next = up[p];
#pragma unroll
      for (int j = 0; j < 4; ++j) m[j] = anc[p][j];
    }
    __syncthreads();
    if (on) {
      up[tid] = next;
#pragma unroll
      for (int j = 0; j < 4; ++j) anc[tid][j] |= m[j];
    }
    __syncthreads();
  }
  if (!invalid && tid < nb) {
    const int row = row0 + tid;
    int slot = -1, pos = 0;
    uint32_t m[4] = {0, 0, 0, 0};
    if (placed) {
      int seen = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m[j] = anc[tid][j];
        seen += __popc(m[j]);
      }
      const int at = hb + tid;
      slot = page_s[at / kPage - col0] * kPage + at % kPage;
      pos = a.prefix_len + hb + seen - 1;
    }
    pos_s[tid] = pos;
    stg(a.slot + row, slot);
    stg(a.position + row, pos);
    stg(a.row_req + row, placed ? b : -1);
#pragma unroll
    for (int j = 0; j < 4; ++j) stg(a.mask + (size_t)row * 4 + j, m[j]);
  }
  __syncthreads();

  // Rotary table: the angle in turns, position theta^(-2j/Dh) / 2 pi, reduced
  // in 64 bits (a far position times an fp32 frequency is off by whole
  // degrees); what is left, in [-1/2, 1/2], is split into an fp32 value and its
  // remainder, which enters to first order.
  const int half = a.Dh / 2, j = tid % half;
  const double turns = exp2(-(2.0 * a.log2_theta / a.Dh) * j) * 0.15915494309189533577;
  for (int i = tid / half; i < nb; i += kThreads / half) {
    const double t = (double)pos_s[i] * turns;
    const double f = t - rint(t);
    const float x = (float)f;
    const float rest = (float)(f - (double)x) * 6.2831853f;
    float sn, cs;
    sincospif(2.0f * x, &sn, &cs);
    float* o = a.rope + ((size_t)(row0 + i) * half + j) * 2;
    stg(o, cs - rest * sn);
    stg(o + 1, sn + rest * cs);
  }
  // Rows behind the last request (all of them if the lengths are not valid).
  const int total = invalid ? 0 : ldg(a.row_start + B);
  for (int row = total + b * kThreads + tid; row < a.N; row += B * kThreads) {
    stg(a.slot + row, -1);
    stg(a.position + row, 0);
    stg(a.row_req + row, -1);
#pragma unroll
    for (int k = 0; k < 4; ++k) stg(a.mask + (size_t)row * 4 + k, 0u);
  }
  for (size_t e = (size_t)total * half + (size_t)b * kThreads + tid; e < (size_t)a.N * half; e += (size_t)B * kThreads) {
    stg(a.rope + 2 * e, 1.0f);
    stg(a.rope + 2 * e + 1, 0.0f);
  }
  if (tid == 0) {
    BatchRequest r;
    r.row0 = row0;
    r.n = placed ? nb : 0;
    r.held = hb;
    r.splits = ns;
    r.part0 = (int)w[2];
    r.pad[0] = r.pad[1] = r.pad[2] = 0;
    stg(a.req + b, r);
    stg(a.status + b, st);
    if (b == 0) {
      stg(a.head + PLAN_UNITS, (int)(invalid ? 0 : w[1]));
      stg(a.head + PLAN_TAKEN, (int)(invalid ? 0 : taken));
      stg(a.head + PLAN_REQUESTS, B);
      stg(a.head + PLAN_ROWS, a.N);
      stg(a.head + PLAN_MAX_PAGES, a.max_pages);
    }
  }
  if (!invalid)
    for (int s = tid; s < ns; s += kThreads) {
      BatchUnit u;
      u.request = b;
      u.run = s;
      u.row0 = row0;
      u.n = placed ? nb : 0;
      u.held = hb;
      u.part0 = (int)w[2];
      u.chunk = (int)chunk;
      u.pad = 0;
      stg(a.units + w[0] + s, u);
    }
}

}  // namespace

hipError_t launch_batch_plan(const PlanArgs& a, hipStream_t st) {
  plan_kernel<<<dim3(a.B), dim3(kThreads), 0, st>>>(a);
  return hipGetLastError();
}

namespace {

// ---------------------------------------------------------------- store
//
// Two kinds of workgroups.  The first turn queries and keys: 256 threads hold the
// cosines and sines of kTurnRows rows (a lane those of 8 dims and their partners
// in the second half, rotate-half pairing) and go through `a.heads_per` heads.
// The others write values: a V row becomes a column of its page, so 64 rows of a
// head meet in LDS, and rows whose slots lie in one aligned piece of eight leave
// together, 16 bytes per dim if there are eight of them.
//
// Bound by bytes, of which V^T's are pieces of lines: 64 trees of up to 31 rows, 32 heads of
// 128 and as many of K/V, take 14 us where the 49 MB stay in the caches and 20 to 26 where they
// do not (2400 to 1900 GB/s); one row each of 512 requests takes 73 to 101 us, two
// bytes of a line per dim and head.  (The values' workgroups first: the same.)
// The norm of queries and keys adds no bytes: a head's 8 or 4 lanes join their sums of
// squares, x / sqrt(mean x^2 + eps) g is turned before anything is rounded, and with gains
// per head the same trees take 15.5 us; 64 prompts of 128 rows, 32 heads on 8, 46 (206 MB,
// 4500 GB/s); 8 single tokens 3.2, launch and latency.
constexpr int kStoreRows = 64;

__device__ __forceinline__ int slot_of(const StoreArgs& a, int row) {
  const int s = row < a.N ? ldg(a.slot + row) : -1;
  return s < a.n_pages * kPage ? s : -1;
}

// 1 / sqrt(mean x^2 + eps) of a head whose dims lie in groups of LANES neighbouring
// lanes, 8 and their partners in each.
template <int LANES>
__device__ __forceinline__ float norm_scale(const float (&u)[8], const float (&v)[8], float eps) {
  float sum = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += u[e] * u[e] + v[e] * v[e];
  sum += dpp_f<kDppQuadXor1>(sum);
  sum += dpp_f<kDppQuadXor2>(sum);
  if (LANES == 8) sum += dpp_f<kDppRowHalfMirror>(sum);
  return rsqrtf(sum * (1.0f / (16 * LANES)) + eps);
}

template <int DH, bool NORM>
__device__ __forceinline__ void turn_rows(const StoreArgs& a, int block, int heads0) {
  constexpr int HALF = DH / 2, LANES = HALF / 8, ROWS = kThreads / LANES;
  const int row = block * ROWS + threadIdx.x / LANES, c = 8 * (threadIdx.x % LANES);
  const int s = slot_of(a, row);
  if (s < 0) return;
  f32x4 cs[4];  // cos, sin of two pairs each
#pragma unroll
  for (int e = 0; e < 4; ++e) cs[e] = ldg((const f32x4*)(a.rope + ((size_t)row * HALF + c) * 2) + e);
  const int heads1 = heads0 + a.heads_per < a.H + a.Hkv ? heads0 + a.heads_per : a.H + a.Hkv;
  // (four heads' loads before the first one's sums: the compiler does not unroll a loop with lane moves)
  constexpr int AHEAD = 4;
  for (int h0 = heads0; h0 < heads1; h0 += AHEAD) {
    bf16x8 p[AHEAD], q[AHEAD], g[AHEAD], w[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int h = h0 + i, kh = h - a.H;
      if (h >= heads1) break;
      const bf16* src = kh < 0 ? a.q + (size_t)row * a.q_stride + (size_t)h * DH : a.k + (size_t)row * a.k_stride + (size_t)kh * DH;
      p[i] = ldg((const bf16x8*)(src + c));
      q[i] = ldg((const bf16x8*)(src + c + HALF));
      const bf16* gain = kh < 0 ? a.q_gain : a.k_gain;
      if (NORM && gain) {
        gain += kh < 0 ? h * a.q_gain_stride : kh * a.k_gain_stride;
        g[i] = ldg((const bf16x8*)(gain + c));
        w[i] = ldg((const bf16x8*)(gain + c + HALF));
      }
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int h = h0 + i, kh = h - a.H;
      if (h >= heads1) break;
      bf16* dst = kh < 0 ? a.q_out + ((size_t)row * a.H + h) * DH
                         : a.k_pages + (((size_t)(s / kPage) * a.Hkv + kh) * kPage + s % kPage) * DH;
      float u[8], v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = bf2f(p[i][e]);
        v[e] = bf2f(q[i][e]);
      }
      if (NORM) {
        const float scale = norm_scale<LANES>(u, v, a.eps);
        const bool gains = (kh < 0 ? a.q_gain : a.k_gain) != nullptr;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] *= scale;
          v[e] *= scale;
          if (gains) {
            u[e] *= bf2f(g[i][e]);
            v[e] *= bf2f(w[i][e]);
          }
        }
      }
      bf16x8 x, y;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float co = cs[e >> 1][2 * (e & 1)], si = cs[e >> 1][2 * (e & 1) + 1];
        x[e] = f2bf(u[e] * co - v[e] * si);
        y[e] = f2bf(v[e] * co + u[e] * si);
      }
      stg((bf16x8*)(dst + c), x);
      stg((bf16x8*)(dst + c + HALF), y);
    }
  }
}

template <int DH>
__device__ __forceinline__ void write_values(const StoreArgs& a, int block, int kh, int part) {
  // (up to seven rows behind the block's own finish its last piece)
  __shared__ int slot_s[kStoreRows + 8];  // from the row before the block on
  __shared__ int piece_s[kStoreRows];     // pieces that begin in the block: first row | rows << 8
  __shared__ int pieces;
  __shared__ int all_whole;               // they are of eight rows each
  __shared__ uint16_t vt[kStoreRows + 7][DH + 2];
  const int r0 = block * kStoreRows, tid = threadIdx.x;
  const int rows = a.N - r0 < kStoreRows + 7 ? a.N - r0 : kStoreRows + 7;
  const int dims = DH / a.dim_parts, d0 = part * dims;  // the workgroup's
  if (tid < kStoreRows + 8) slot_s[tid] = r0 + tid > 0 ? slot_of(a, r0 + tid - 1) : -1;
#pragma unroll 4
  for (int e = tid; e < rows * (dims / 8); e += kThreads) {
    const int i = e / (dims / 8), c = d0 + 8 * (e % (dims / 8));
    const bf16x8 v = ldg((const bf16x8*)(a.v + ((size_t)r0 + i) * a.v_stride + (size_t)kh * DH + c));
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bf16 x = v[u];  // (a bit cast of the vector's element itself takes element 0)
      vt[i][c + u] = __builtin_bit_cast(uint16_t, x);
    }
  }
  __syncthreads();
  if (tid < kStoreRows) {  // (one wave)
    const int s = slot_s[tid + 1];
    const bool begins = s >= 0 && ((s & 7) == 0 || slot_s[tid] != s - 1);
    int n = 1;
    while (n < 8 && (s & 7) + n < 8 && slot_s[tid + 1 + n] == s + n) ++n;
    const uint64_t all = __ballot(begins);
    if (begins) piece_s[__popcll(all & ((1ull << tid) - 1))] = tid | n << 8;
    const uint64_t parts = __ballot(begins && n < 8);
    if (tid == 0) {
      pieces = __popcll(all);
      all_whole = parts == 0;
    }
  }
  __syncthreads();
  const auto write_piece = [&](int piece, int c, bool whole) {
    const int p = piece_s[piece], i = p & 0xff, n = whole ? 8 : p >> 8, s = slot_s[i + 1];
    uint16_t* dst = (uint16_t*)a.v_pages + (((size_t)(s / kPage) * a.Hkv + kh) * DH + c) * kPage + s % kPage;
    if (n == 8) {
      bf16x8 v;
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = __builtin_bit_cast(bf16, vt[i + u][c]);
      stg((bf16x8*)dst, v);
      return;
    }
    // (part of a piece: its entries in the largest aligned groups)
    for (int u = 0; u < n;) {
      const int at = (s & 7) + u;
      if ((at & 3) == 0 && u + 4 <= n) {
        stg((uint2*)(dst + u), make_uint2((uint32_t)vt[i + u][c] | (uint32_t)vt[i + u + 1][c] << 16,
                                          (uint32_t)vt[i + u + 2][c] | (uint32_t)vt[i + u + 3][c] << 16));
        u += 4;
      } else if ((at & 1) == 0 && u + 2 <= n) {
        stg((uint32_t*)(dst + u), (uint32_t)vt[i + u][c] | (uint32_t)vt[i + u + 1][c] << 16);
        u += 2;
      } else {
        stg(dst + u, vt[i + u][c]);
        u += 1;
      }
    }
  };
  // Whole pieces go line by line (64 prompts of 128 rows, 8 K/V heads: 46 us for 48), parts
  // dim by dim (64 trees of up to 31 rows, 32 heads: 14.3 for 15.8).
  if (all_whole) {
    for (int e = tid; e < pieces * dims; e += kThreads) write_piece(e % pieces, d0 + e / pieces, true);
  } else {
    for (int e = tid; e < pieces * dims; e += kThreads) write_piece(e / dims, d0 + e % dims, false);
  }
}

template <int DH, bool NORM>
__global__ __launch_bounds__(kThreads) void store_kernel(StoreArgs a, int turn_blocks, int head_blocks) {
  if (!plan_is_for(a.head, a.B, a.N)) return;
  const int x = blockIdx.x, turns = turn_blocks * head_blocks;
  if (x < turns)
    turn_rows<DH, NORM>(a, x % turn_blocks, x / turn_blocks * a.heads_per);
  else
    write_values<DH>(a, (x - turns) / a.dim_parts / a.Hkv, (x - turns) / a.dim_parts % a.Hkv, (x - turns) % a.dim_parts);
}

// ---------------------------------------------------------------- rollback
//
// As llmcad_commit_path, in pages.  Accepted row path[k] moves to row k, and
// path[k] > k: a row may be written only after the moves of smaller k have read it.
// A K row's 16-byte piece is one thread's, which makes the moves in the order of k
// (in batches: eight loads, then their eight stores).  A dim of V^T is a line of
// its page with an entry per move: as many lanes of one wave as there are moves
// read theirs in one instruction, and write them after it, several dims in flight.
//
// Chains are in place: a workgroup that finds no move ends (32 requests, 32 layers,
// 32 heads of 128: 8 us, the launch).  49 moves of 22 such requests' trees take 178 us:
// an entry per dim costs a 128-byte line's read and a 32-byte write (430 MB and 110
// MB, 3 TB/s with such writes), which is the price of V^T's layout; K's rows are 26
// MB each way.
constexpr int kCommitBatch = 8;

__device__ __forceinline__ void move_keys(bf16x8* base, size_t page_step, int slot_step, const int* src, const int* dst, int moves) {
  for (int k0 = 0; k0 < moves; k0 += kCommitBatch) {
    bf16x8 v[kCommitBatch];
#pragma unroll
    for (int u = 0; u < kCommitBatch; ++u)
      if (k0 + u < moves) v[u] = ldg(base + (size_t)(src[k0 + u] / kPage) * page_step + (src[k0 + u] % kPage) * slot_step);
#pragma unroll
    for (int u = 0; u < kCommitBatch; ++u)
      if (k0 + u < moves) stg(base + (size_t)(dst[k0 + u] / kPage) * page_step + (dst[k0 + u] % kPage) * slot_step, v[u]);
  }
}

// V^T entries of `dims` dims from base on (lines of kPage entries), `moves` entries
// of each: REACH per lane.
template <int REACH>
__device__ __forceinline__ void move_values(uint16_t* base, size_t page_step, const int* src, const int* dst, int moves, int dims) {
  constexpr int AHEAD = 8 / REACH;
  int lanes = 1;  // per dim
  while (lanes * REACH < moves) lanes *= 2;
  const int k = threadIdx.x % lanes, step = kThreads / lanes;
  size_t from[REACH], to[REACH];
#pragma unroll
  for (int i = 0; i < REACH; ++i) {
    const int m = k + i * lanes < moves ? k + i * lanes : 0;
    from[i] = (size_t)(src[m] / kPage) * page_step + src[m] % kPage;
    to[i] = (size_t)(dst[m] / kPage) * page_step + dst[m] % kPage;
  }
  for (int d0 = threadIdx.x / lanes; d0 < dims; d0 += AHEAD * step) {
    uint16_t v[AHEAD][REACH];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int i = 0; i < REACH; ++i)
        if (d0 + u * step < dims && k + i * lanes < moves) v[u][i] = ldg(base + (size_t)(d0 + u * step) * kPage + from[i]);
    __builtin_amdgcn_wave_barrier();  // (no store moves before a load: another lane may read what it overwrites)
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
#pragma unroll
      for (int i = 0; i < REACH; ++i)
        if (d0 + u * step < dims && k + i * lanes < moves) stg(base + (size_t)(d0 + u * step) * kPage + to[i], v[u][i]);
  }
}

// A workgroup per request and a.heads_per neighbouring K/V heads of a layer.
__global__ __launch_bounds__(kThreads) void commit_kernel(CommitArgs a) {
  __shared__ int src_s[128], dst_s[128], moves_s[2];  // slots of the moves, in the order of k
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, dh = a.Dh;
  const BatchRequest r = ldg(a.req + b);
  const int len = ldg(a.accept_len + b);
  if (!plan_is_for(a.head, a.B, a.N)) return;
  if (len < 1 || len >= r.n) return;  // (nothing moves, or not the outcome of a tree of n rows)
  const int limit = a.n_pages * kPage;
  int src = -1, dst = -1;
  if (tid < len) {
    const int k = tid + 1, p = ldg(a.path + r.row0 + k);
    dst = ldg(a.slot + r.row0 + k);
    src = p > k && p < r.n ? ldg(a.slot + r.row0 + p) : -1;  // (in place already, or no row of the tree)
  }
  const bool moves_here = src >= 0 && src < limit && dst >= 0 && dst < limit;
  const uint64_t all = __ballot(moves_here);
  if (lane == 0 && wave < 2) moves_s[wave] = __popcll(all);
  __syncthreads();
  const int moves = moves_s[0] + moves_s[1];
  if (moves == 0) return;
  if (moves_here) {
    const int at = __popcll(all & ((1ull << lane) - 1)) + (wave == 1 ? moves_s[0] : 0);
    src_s[at] = src;
    dst_s[at] = dst;
  }
  __syncthreads();
  const size_t page = (size_t)a.Hkv * kPage * dh;  // elements of a page
  const int groups = up_div(a.Hkv, a.heads_per), layer = blockIdx.x / groups, kh0 = blockIdx.x % groups * a.heads_per;
  const int heads = a.Hkv - kh0 < a.heads_per ? a.Hkv - kh0 : a.heads_per;
  const size_t at = (size_t)layer * a.n_pages * page + (size_t)kh0 * kPage * dh;
  const int kp = dh / 8;  // pieces of a K row
  for (int e = tid; e < heads * kp; e += kThreads)
    move_keys((bf16x8*)(a.k_pages + at + (size_t)(e / kp) * kPage * dh) + e % kp, page / 8, kp, src_s, dst_s, moves);
  uint16_t* values = (uint16_t*)(a.v_pages + at);
  if (moves <= 64)
    move_values<1>(values, page, src_s, dst_s, moves, heads * dh);
  else
    move_values<2>(values, page, src_s, dst_s, moves, heads * dh);
}

}  // namespace

namespace {

template <bool NORM>
hipError_t launch_store(const StoreArgs& args, hipStream_t st) {
  StoreArgs a = args;
  const int turn_blocks = cdiv(a.N, kThreads / (a.Dh / 16)), heads = a.H + a.Hkv;
  // heads per workgroup: a table row for up to eight, if about 128 workgroups are left (64
  // trees of 31, 64 heads: 16.9 us with one head, 15.0 with eight)
  a.heads_per = (int)((long long)turn_blocks * heads / 128);
  a.heads_per = a.heads_per < 1 ? 1 : a.heads_per > 8 ? 8 : a.heads_per;
  const int head_blocks = cdiv(heads, a.heads_per);
  const long long values = (long long)cdiv(a.N, kStoreRows) * a.Hkv;
  // A head's values are shared until there are 256 workgroups (68 single rows of 8 heads: 14.5 us
  // with one each, 5.2 so; with 1024 wanted, 152 requests of 3 rows and 32 heads take 18.5 for 13.8).
  a.dim_parts = 1;
  while (a.dim_parts < 8 && values * a.dim_parts < 256) a.dim_parts *= 2;
  const dim3 grid((unsigned)(turn_blocks * head_blocks + values * a.dim_parts));
  if (a.Dh == 128)
    store_kernel<128, NORM><<<grid, dim3(kThreads), 0, st>>>(a, turn_blocks, head_blocks);
  else
    store_kernel<64, NORM><<<grid, dim3(kThreads), 0, st>>>(a, turn_blocks, head_blocks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_batch_store(const StoreArgs& a, hipStream_t st) { return launch_store<false>(a, st); }
hipError_t launch_batch_norm_store(const StoreArgs& a, hipStream_t st) { return launch_store<true>(a, st); }

hipError_t launch_batch_commit(const CommitArgs& args, hipStream_t st) {
  CommitArgs a = args;
  // heads per workgroup: up to eight, if about 2048 workgroups are left
  const long long heads = (long long)a.B * a.L * a.Hkv;
  a.heads_per = (int)(heads / 2048 < 1 ? 1 : heads / 2048 > 8 ? 8 : heads / 2048);
  commit_kernel<<<dim3(a.L * cdiv(a.Hkv, a.heads_per), a.B), dim3(kThreads), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace llmcad
