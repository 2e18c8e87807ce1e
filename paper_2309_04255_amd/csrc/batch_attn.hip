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

// Workgroup (x, y): K/V head y, run x of keys: the first KP x `blocks` (row blocks of
// all rows; 0 if wide_kernel has the prefix) take the prefix's key splits, the others the plan's runs of pages, one
// block of 16 (row, query head) pairs after the other.  The four waves take
// every fourth 32-key step and meet in LDS.
template <int DH>
__global__ __launch_bounds__(kThreads) void split_kernel(AttnArgs a, int blocks) {
  __shared__ float o_s[kWaves][16][DH + 4];
  __shared__ float ml_s[kWaves][16][2];
  constexpr int NS = KeyStep<DH>::NS, NB = KeyStep<DH>::NB;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, g = lane >> 4, wave = wave_index();
  const int kh = blockIdx.y, group = a.H / a.Hkv;
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

// The prefix for many rows: 128 (row, query head) pairs of a K/V head per
// workgroup, 32 per wave, over one key split.  Tiles of 64 keys are shared
// through LDS in fragment order (every access is 16 bytes per lane, lane by
// lane): while a tile is computed the next one is on its way to registers, and
// it goes to the other buffer before the barrier.
//
// The running maximum is only a reference point: any value near it serves, so
// the output is rescaled only when some score exceeds it by 2^kSlack, and
// until then no lane needs another's scores.  The sums are per lane, joined at
// the end.  Probabilities (up to 2^kSlack) enter the value product in bf16, half
// a step of 2^-8 each.
constexpr int kTileKeys = 64;
constexpr int kTileRows = 128;
constexpr float kSlack = 8.0f;

template <int DH>
__global__ __launch_bounds__(kThreads, 2) void wide_kernel(AttnArgs a) {
  constexpr int NS = KeyStep<DH>::NS, NB = KeyStep<DH>::NB, LOADS = KeyStep<DH>::LOADS;
  constexpr int PER = LOADS / 2;  // fragments per wave and tile: K of a step, or V^T of a step
  constexpr int TILE = 2 * LOADS * 1024;
  __shared__ __align__(16) char lds[2][TILE];
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4, wave = wave_index();
  const int group = a.H / a.Hkv, pairs = a.N * group, tiles = up_div(pairs, kTileRows);
  // workgroup w runs on XCD w % 8: each XCD gets a contiguous share of the units,
  // tile by tile of one (head, split), so that its keys are read into one L2
  const int units = tiles * a.KP * a.Hkv, per_xcd = up_div(units, 8);
  const int u = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per_xcd || u >= units) return;
  const int tile = u % tiles, split = u / tiles % a.KP, kh = u / tiles / a.KP;
  const int ktiles = up_div(a.P, kTileKeys), per = up_div(ktiles, a.KP);
  const int first = split * per, last = first + per < ktiles ? first + per : ktiles;

  bf16x8 qf[2][NS];
#pragma unroll
  for (int rb = 0; rb < 2; ++rb) {
    const int pr0 = tile * kTileRows + wave * 32 + rb * 16 + li, pr = pr0 < pairs ? pr0 : pairs - 1;
    const bf16* q = a.q + (size_t)(pr / group) * a.q_stride + (size_t)(kh * group + pr % group) * DH + 8 * g;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[rb][s] = ldg((const bf16x8*)(q + 32 * s));
  }
  // this wave's part of a tile: waves 0 and 2 the keys of its two steps, 1 and 3 the values
  const bool values = (wave & 1) != 0;
  const int key = 32 * (wave >> 1);
  const bf16* src = values ? a.vc + ((size_t)kh * DH + li) * a.cap + key + 8 * g + (size_t)first * kTileKeys
                           : a.kc + ((size_t)kh * a.cap + key + 8 * (li >> 2) + (li & 3) + (size_t)first * kTileKeys) * DH + 8 * g;
  const size_t advance = values ? kTileKeys : (size_t)kTileKeys * DH;
  const int lds_at = ((wave >> 1) * LOADS + (values ? 2 * NS : 0)) * 1024 + lane * 16;
  bf16x8 stage[PER];
  auto fetch = [&]() {
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const size_t off = values ? (size_t)e * 16 * a.cap : (size_t)((e / NS) * 4 * DH + (e % NS) * 32);
      stage[e] = ldg((const bf16x8*)(src + off));
    }
    src += advance;
  };
  auto put = [&](int t) {  // (tile t)
    char* at = lds[t & 1] + lds_at;
    const int valid = a.P - (t * kTileKeys + key + 8 * g);  // (values of keys past the prefix: zeros)
    if (values && (t + 1) * kTileKeys > a.P) {
#pragma unroll
      for (int e = 0; e < PER; ++e)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= valid) stage[e][i] = (bf16)0.0f;
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) lds_st<bf16x8>(at + e * 1024, stage[e]);
  };

  float m[2], neg_m[2], l[2];
  f32x4 o[2][NB];
#pragma unroll
  for (int rb = 0; rb < 2; ++rb) {
    m[rb] = -INFINITY;
    neg_m[rb] = 0.0f;
    l[rb] = 0.0f;
#pragma unroll
    for (int db = 0; db < NB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  if (first < last) {
    fetch();
    put(first);
  }
  __syncthreads();
  for (int t = first; t < last; ++t) {
    if (t + 1 < last) fetch();
    const char* at = lds[t & 1] + lane * 16;
    f32x4 sc[2][4];  // [row block][step, key block]
#pragma unroll
    for (int sb = 0; sb < 4; ++sb) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) sc[rb][sb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const bf16x8 k = lds_ld<bf16x8>(at + ((sb >> 1) * LOADS + (sb & 1) * NS + s) * 1024);
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) sc[rb][sb] = mfma16x16x32(k, qf[rb][s], sc[rb][sb]);
      }
    }
    if ((t + 1) * kTileKeys > a.P) {
      const int valid = a.P - t * kTileKeys;
#pragma unroll
      for (int sb = 0; sb < 4; ++sb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (32 * (sb >> 1) + 8 * g + 4 * (sb & 1) + i >= valid)
#pragma unroll
            for (int rb = 0; rb < 2; ++rb) sc[rb][sb][i] = -INFINITY;
    }
    float mx[2];
    bool grow = false;
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
      mx[rb] = sc[rb][0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx[rb] = fmaxf(mx[rb], sc[rb][e >> 2][e & 3]);
      mx[rb] *= a.scale_log2;
      grow |= mx[rb] > m[rb] + kSlack;
    }
    if (__any(grow)) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        const float m_new = fmaxf(m[rb], col4_max(mx[rb]));
        const float m_use = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m[rb] - m_use);
        m[rb] = m_new;
        neg_m[rb] = -m_use;
        l[rb] *= alpha;
#pragma unroll
        for (int db = 0; db < NB; ++db) o[rb][db] = o[rb][db] * alpha;
      }
    }
    bf16x8 p[2][2];
#pragma unroll
    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[rb][e >> 2][e & 3], a.scale_log2, neg_m[rb]));
        l[rb] += v;
        p[rb][e >> 3][e & 7] = f2bf(v);
      }
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int db = 0; db < NB; ++db) {
        const bf16x8 v = lds_ld<bf16x8>(at + (st * LOADS + 2 * NS + db) * 1024);
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) o[rb][db] = mfma16x16x32(v, p[rb][st], o[rb][db]);
      }
    if (t + 1 < last) put(t + 1);
    __syncthreads();
  }
#pragma unroll
  for (int rb = 0; rb < 2; ++rb) {
    const int pr = tile * kTileRows + wave * 32 + rb * 16 + li;
    const float sum = col4_sum(l[rb]);
    if (pr >= pairs) continue;
    const size_t at = ((size_t)split * a.N + pr / group) * a.H + kh * group + pr % group;
#pragma unroll
    for (int db = 0; db < NB; ++db) stg((f32x4*)(a.part_o + at * DH + 16 * db + 4 * g), o[rb][db]);
    if (g == 0) {
      stg(a.part_ml + at * 2, m[rb]);
      stg(a.part_ml + at * 2 + 1, sum);
    }
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

// Few pairs of rows and heads per K/V head: the waves share 16 of them and split the keys; many:
// the waves split the pairs and share the keys.
static bool wide_prefix(int N, int H, int Hkv) { return (long long)N * (H / Hkv) > 64; }

int prefix_splits(int N, int H, int Hkv, int P) {
  if (P <= 0) return 0;
  int KP, most;
  if (wide_prefix(N, H, Hkv)) {
    KP = 512 / (cdiv(N * (H / Hkv), kTileRows) * Hkv);
    most = cdiv(P, 2 * kTileKeys);
  } else {
    KP = cdiv(512, cdiv(N * (H / Hkv), 16) * Hkv);
    most = cdiv(P, 128);
  }
  if (KP > most) KP = most;
  if (KP > max_prefix_splits(N)) KP = max_prefix_splits(N);
  return KP < 1 ? 1 : KP;
}

template <int DH>
static hipError_t launch_attention(const AttnArgs& a, hipStream_t st) {
  const int group = a.H / a.Hkv;
  const bool wide = a.KP > 0 && wide_prefix(a.N, a.H, a.Hkv);
  const int blocks = wide || a.KP == 0 ? 0 : cdiv(a.N * group, 16);
  const long long most = (long long)a.B * cdiv(a.max_pages, 2);  // (a run has two pages or more)
  const int units = most < plan_max_units(a.B) ? (int)most : plan_max_units(a.B);
  if (wide) {
    const int wu = cdiv(a.N * group, kTileRows) * a.KP * a.Hkv;
    wide_kernel<DH><<<dim3(cdiv(wu, 8) * 8), dim3(kThreads), 0, st>>>(a);
  }
  split_kernel<DH><<<dim3(a.KP * blocks + units, a.Hkv), dim3(kThreads), 0, st>>>(a, blocks);
  join_kernel<DH><<<dim3((unsigned)(((long long)a.N * a.H + kWaves - 1) / kWaves)), dim3(kThreads), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_batch_attention(const AttnArgs& a, hipStream_t st) {
  return a.Dh == 128 ? launch_attention<128>(a, st) : launch_attention<64>(a, st);
}

}  // namespace llmcad
