// Attention of several requests' rows to the prefix they share, to their own
// pages and to their own branch.
//
//   out[r][h] = sum_t softmax_t(q[r][h] . K[t] / sqrt(Dh)) V[t]
//
// over the prefix [0, P), the tokens its request holds and the rows of the
// request that its mask names.  The prefix's keys and values are read for all
// requests at once; a request's own for its rows at once.  Both leave partial
// results (maximum, sum, unnormalised output), which a second launch joins.
//
// As in the verification pass, S^T = K q^T and O^T = V^T P^T run on the matrix
// cores with K and V^T taken from memory in fragment order: K block b of a
// 32-key step puts key 8 (r / 4) + 4 b + r % 4 in its row r, so that the lane
// that holds a score also holds the value operand's slot for that key.
#include "batch.h"

namespace llmcad {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;

__device__ __forceinline__ int up_div(int x, int a) { return (x + a - 1) / a; }

// One 32-key step's operands of a wave: K block b, 32-dim step s at f[b NS + s],
// V^T 16-dim block db at f[2 NS + db].
template <int DH>
struct KeyStep {
  static constexpr int NS = DH / 32, NB = DH / 16, LOADS = 2 * NS + NB;
  bf16x8 f[LOADS];
};

// k: K row of the step's first key (rows DH apart); vt: its entry in V^T row 0
// (rows vs apart).
template <int DH>
__device__ __forceinline__ void load_step(KeyStep<DH>& R, const bf16* k, const bf16* vt, int vs) {
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4;
  constexpr int NS = KeyStep<DH>::NS, NB = KeyStep<DH>::NB;
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int s = 0; s < NS; ++s)
      R.f[b * NS + s] = ldg((const bf16x8*)(k + (size_t)(8 * (li >> 2) + 4 * b + (li & 3)) * DH + 32 * s + 8 * g));
#pragma unroll
  for (int db = 0; db < NB; ++db) R.f[2 * NS + db] = ldg((const bf16x8*)(vt + (size_t)(16 * db + li) * vs + 8 * g));
}

// Running softmax of 16 rows: lane (li, g) holds row li's maximum and sum, and
// dims 16 db + 4 g + i of its output.
template <int DH>
struct RowState {
  float m, l;
  f32x4 o[DH / 16];
};

// One step for 16 rows.  vis: bit e set if the lane's row sees key 8 g + e; p:
// the lane's probabilities against the new maximum.
template <int DH>
__device__ __forceinline__ void attend(const KeyStep<DH>& R, const bf16x8 (&qf)[DH / 32], uint32_t vis, float scale_log2,
                                       RowState<DH>& st, float (&p)[8]) {
  constexpr int NS = KeyStep<DH>::NS, NB = KeyStep<DH>::NB;
  f32x4 sc[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    sc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < NS; ++s) sc[b] = mfma16x16x32(R.f[b * NS + s], qf[s], sc[b]);
  }
  float sv[8], mx = -INFINITY;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sv[e] = (vis >> e) & 1u ? sc[e >> 2][e & 3] * scale_log2 : -INFINITY;
    mx = fmaxf(mx, sv[e]);
  }
  mx = col4_max(mx);
  const float m_new = fmaxf(st.m, mx);
  const float m_use = m_new == -INFINITY ? 0.0f : m_new;
  const float alpha = __builtin_amdgcn_exp2f(st.m - m_use);
  bf16x8 ph, pl;
  float sum = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = __builtin_amdgcn_exp2f(sv[e] - m_use);
    ph[e] = f2bf(p[e]);
    pl[e] = f2bf(p[e] - bf2f(ph[e]));
    sum += p[e];
  }
  st.l = st.l * alpha + col4_sum(sum);
  st.m = m_new;
#pragma unroll
  for (int db = 0; db < NB; ++db) {
    st.o[db] = st.o[db] * alpha;
    st.o[db] = mfma16x16x32(R.f[2 * NS + db], ph, st.o[db]);
    st.o[db] = mfma16x16x32(R.f[2 * NS + db], pl, st.o[db]);
  }
}

// Values of keys that no row may read count as zeros (0 x NaN is NaN): the
// lane's keys 8 g + e with e >= valid.
template <int DH>
__device__ __forceinline__ void clear_values(KeyStep<DH>& R, int valid) {
#pragma unroll
  for (int db = 0; db < KeyStep<DH>::NB; ++db)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e >= valid) R.f[2 * KeyStep<DH>::NS + db][e] = (bf16)0.0f;
}

// A step whose keys some rows see and others do not: an Inf or NaN among its
// values would reach the others as 0 x Inf.  Such values are left out of the
// product (true: there are some)...
template <int DH>
__device__ __forceinline__ bool take_out_nonfinite(KeyStep<DH>& R, KeyStep<DH>& taken) {
  bool any = false;
#pragma unroll
  for (int db = 0; db < KeyStep<DH>::NB; ++db)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bf16 v = R.f[2 * KeyStep<DH>::NS + db][e];
      any |= (__builtin_bit_cast(uint16_t, v) & 0x7f80) == 0x7f80;
    }
  if (!__any(any)) return false;
#pragma unroll
  for (int db = 0; db < KeyStep<DH>::NB; ++db)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int f = 2 * KeyStep<DH>::NS + db;
      const bf16 v = R.f[f][e];
      const bool bad = (__builtin_bit_cast(uint16_t, v) & 0x7f80) == 0x7f80;
      taken.f[f][e] = bad ? v : (bf16)0.0f;
      if (bad) R.f[f][e] = (bf16)0.0f;
    }
  return true;
}
// ... and added for the rows that see them: the value of dim 16 db + 4 g + i at
// key 8 k + e is held by lane (4 g + i, k), row li's probability by lane (li, k).
template <int DH>
__device__ __forceinline__ void add_nonfinite(const KeyStep<DH>& taken, uint32_t vis, const float (&p)[8], RowState<DH>& st) {
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4;
#pragma unroll 1
  for (int k = 0; k < 4; ++k) {
    const uint32_t sees = (uint32_t)__shfl((int)vis, 16 * k + li, kWave);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float pe = __shfl(p[e], 16 * k + li, kWave);
#pragma unroll
      for (int db = 0; db < KeyStep<DH>::NB; ++db) {
        const float mine = bf2f(taken.f[2 * KeyStep<DH>::NS + db][e]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float v = __shfl(mine, 16 * k + 4 * g + i, kWave);
          if (((sees >> e) & 1u) && v != 0.0f) st.o[db][i] += pe * v;
        }
      }
    }
  }
}

// Workgroup (x, y): K/V head y, run x of keys: the first KP x (row blocks of all
// rows) take the prefix's key splits, the others the plan's runs of pages, one
// block of 16 (row, query head) pairs after the other.  The four waves take
// every fourth 32-key step and meet in LDS.
template <int DH>
__global__ __launch_bounds__(kThreads) void split_kernel(AttnArgs a) {
  __shared__ float o_s[kWaves][16][DH + 4];
  __shared__ float ml_s[kWaves][16][2];
  constexpr int NS = KeyStep<DH>::NS, NB = KeyStep<DH>::NB;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, g = lane >> 4, wave = wave_index();
  const int kh = blockIdx.y, group = a.H / a.Hkv;
  const int blocks = (int)(((long long)a.N * group + 15) / 16);
  int x = blockIdx.x;
  const bool prefix = x < a.KP * blocks;
  int row0, n, held = 0, lim, first, last;  // rows, visible key range, steps [first, last)
  size_t part;                              // partial row of row 0
  const int* table = nullptr;
  if (prefix) {
    const int split = x / blocks;
    row0 = 0;
    n = a.N;
    lim = a.P;
    const int steps = up_div(a.P, 32), per = up_div(steps, a.KP);
    first = split * per;
    last = first + per < steps ? first + per : steps;
    part = (size_t)split * a.N;
  } else {
    x -= a.KP * blocks;
    if (x >= ldg(a.head + PLAN_UNITS)) return;
    const int u = ldg(a.units + x);
    const BatchRequest r = ldg(a.req + (u >> 16));
    if (r.n == 0) return;
    const int run = u & 0xffff, chunk = ldg(a.head + PLAN_CHUNK);
    row0 = r.row0;
    n = r.n;
    held = r.held;
    lim = r.held + r.n;
    table = a.table + (size_t)(u >> 16) * a.max_pages;
    const int room = a.max_pages < (1 << 25) ? a.max_pages * 2 : 1 << 26;  // (steps of the table)
    const int steps = up_div(lim, 32) < room ? up_div(lim, 32) : room;
    const long long f = (long long)run * chunk * 2, t = f + (long long)chunk * 2;
    first = f < steps ? (int)f : steps;
    last = t < steps ? (int)t : steps;
    part = (size_t)a.KP * a.N + r.part0 + (size_t)run * r.n;
  }
  const int pairs = n * group;
  const int b0 = prefix ? x % blocks : 0, b1 = prefix ? b0 + 1 : up_div(pairs, 16);
  for (int blk = b0; blk < b1; ++blk) {
    const int pr = 16 * blk + li < pairs ? 16 * blk + li : pairs - 1;
    const size_t row = (size_t)row0 + pr / group;
    const int head = kh * group + pr % group;
    bf16x8 qf[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = ldg((const bf16x8*)(a.q + row * a.q_stride + (size_t)head * DH + 32 * s + 8 * g));
    uint32_t anc[4] = {0, 0, 0, 0};
    if (!prefix)
#pragma unroll
      for (int j = 0; j < 4; ++j) anc[j] = ldg(a.mask + row * 4 + j);
    RowState<DH> st;
    st.m = -INFINITY;
    st.l = 0.0f;
#pragma unroll
    for (int db = 0; db < NB; ++db) st.o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int j = first + wave; j < last; j += kWaves) {
      const int key0 = 32 * j;
      KeyStep<DH> R;
      if (prefix) {
        load_step<DH>(R, a.kc + ((size_t)kh * a.cap + key0) * DH, a.vc + (size_t)kh * DH * a.cap + key0, a.cap);
      } else {
        const int id = wave_uniform(ldg(table + key0 / kPage));
        if (id < 0 || id >= a.n_pages) continue;
        const size_t page = ((size_t)id * a.Hkv + kh) * kPage * DH;
        load_step<DH>(R, a.kp + page + (size_t)(key0 % kPage) * DH, a.vp + page + key0 % kPage, kPage);
      }
      uint32_t vis = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = key0 + 8 * g + e;
        bool sees = key < lim;
        if (!prefix && key >= held) {
          const int t = key - held;
          sees = sees && t < LLMCAD_MAX_NODES && ((anc[(t >> 5) & 3] >> (t & 31)) & 1u);
        }
        vis |= sees ? 1u << e : 0u;
      }
      if (key0 + 32 > lim) clear_values<DH>(R, lim - (key0 + 8 * g));
      float pr_[8];
      if (!prefix && key0 + 32 > held) {
        KeyStep<DH> taken;
        const bool some = take_out_nonfinite<DH>(R, taken);
        attend<DH>(R, qf, vis, a.scale_log2, st, pr_);
        if (some) add_nonfinite<DH>(taken, vis, pr_, st);
      } else {
        attend<DH>(R, qf, vis, a.scale_log2, st, pr_);
      }
    }
    // the four waves' states, joined in wave order
    __syncthreads();
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) o_s[wave][li][16 * db + 4 * g + i] = st.o[db][i];
    if (g == 0) {
      ml_s[wave][li][0] = st.m;
      ml_s[wave][li][1] = st.l;
    }
    __syncthreads();
    for (int e = tid; e < 16 * DH; e += kThreads) {
      const int i = e / DH, c = e % DH, p = 16 * blk + i;
      if (p >= pairs) continue;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml_s[w][i][0]);
      const float mu = m == -INFINITY ? 0.0f : m;
      float l = 0.0f, o = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml_s[w][i][0] - mu);
        l += f * ml_s[w][i][1];
        o += f * o_s[w][i][c];
      }
      const size_t at = (part + p / group) * a.H + kh * group + p % group;
      stg(a.part_o + at * DH + c, o);
      if (c == 0) {
        stg(a.part_ml + at * 2, m);
        stg(a.part_ml + at * 2 + 1, l);
      }
    }
    __syncthreads();
  }
}

// A wave per (row, head): its partial results in the order of their keys.
template <int DH>
__global__ __launch_bounds__(kThreads) void join_kernel(AttnArgs a) {
  const size_t item = (size_t)blockIdx.x * kWaves + wave_index();
  const int lane = threadIdx.x & 63;
  if (item >= (size_t)a.N * a.H) return;
  const int row = (int)(item / a.H), h = (int)(item % a.H);
  const int b = ldg(a.row_req + row);
  if (b < 0) return;  // (no request's row: left as it was)
  const BatchRequest r = ldg(a.req + b);
  const int parts = a.KP + r.splits;
  constexpr int PER = DH / 64;
  float m = -INFINITY, l = 0.0f, o[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) o[i] = 0.0f;
  for (int p = 0; p < parts; ++p) {
    const size_t pr = p < a.KP ? (size_t)p * a.N + row
                               : (size_t)a.KP * a.N + r.part0 + (size_t)(p - a.KP) * r.n + (row - r.row0);
    const size_t at = pr * a.H + h;
    const float pm = ldg(a.part_ml + at * 2), pl = ldg(a.part_ml + at * 2 + 1);
    const float mm = fmaxf(m, pm), mu = mm == -INFINITY ? 0.0f : mm;
    const float fa = __builtin_amdgcn_exp2f(m - mu), fb = __builtin_amdgcn_exp2f(pm - mu);
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] = fa * o[i] + fb * ldg(a.part_o + at * DH + lane * PER + i);
    l = fa * l + fb * pl;
    m = mm;
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < PER; ++i) stg(a.out + item * DH + lane * PER + i, f2bf(o[i] * inv));
}

}  // namespace

int prefix_splits(int N, int H, int Hkv, int P) {
  if (P <= 0) return 0;
  const int steps = cdiv(P, 32), tiles = cdiv(N * (H / Hkv), 16) * Hkv;
  int KP = cdiv(512, tiles);
  if (KP > cdiv(steps, 4)) KP = cdiv(steps, 4);
  if (KP > max_prefix_splits(N)) KP = max_prefix_splits(N);
  return KP < 1 ? 1 : KP;
}

hipError_t launch_batch_attention(const AttnArgs& a, hipStream_t st) {
  const int blocks = (int)(((long long)a.N * (a.H / a.Hkv) + 15) / 16);
  const long long most = (long long)a.B * cdiv(a.max_pages, 2);  // (a run has two pages or more)
  const int units = most < plan_max_units(a.B) ? (int)most : plan_max_units(a.B);
  const dim3 grid(a.KP * blocks + units, a.Hkv);
  const dim3 join((unsigned)(((long long)a.N * a.H + kWaves - 1) / kWaves));
  if (a.Dh == 128) {
    split_kernel<128><<<grid, dim3(kThreads), 0, st>>>(a);
    join_kernel<128><<<join, dim3(kThreads), 0, st>>>(a);
  } else {
    split_kernel<64><<<grid, dim3(kThreads), 0, st>>>(a);
    join_kernel<64><<<join, dim3(kThreads), 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace llmcad
