// Attention of several requests' rows to the prefix they share, to their own
// pages and to their own branch.
//
//   out[r][h] = sum_t softmax_t(q[r][h] . K[t] / sqrt(Dh)) V[t]
//
// over the prefix [0, P), the tokens its request holds and the rows of the
// request that its mask names.  The prefix's keys and values are read for all
// requests at once; a request's own for its rows at once.  Every workgroup
// takes a run of keys for some (row, query head) pairs of one K/V head and
// leaves partial results (maximum, sum, unnormalised output), which a second
// launch joins.
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
constexpr int kTileKeys = kPage;  // keys of a tile: two 32-key steps, one page
constexpr float kSlack = 8.0f;

__device__ __forceinline__ int up_div(int x, int a) { return (x + a - 1) / a; }

// Fragments of a 32-key step: K block b, 32-dim step s at b NS + s; V^T 16-dim
// block db at 2 NS + db.
template <int DH>
struct Frags {
  static constexpr int NS = DH / 32, NB = DH / 16, LOADS = 2 * NS + NB;
};

// What a workgroup works on.
struct Unit {
  int kh;            // K/V head
  int row0, pairs;   // first row, (row, query head of the group) pairs
  int pair0;         // first pair of a tile unit
  int first, last;   // tiles of kTileKeys keys
  int lim;           // keys at or past it are not there
  int held;          // keys from it on are the request's rows, seen by mask (the prefix: lim)
  const int* table;  // pages, or null: the prefix
  size_t part;       // partial row of row0
};

// Where a tile's keys and values lie: K rows of the head DH apart, V^T rows vs.
struct TileAt {
  const bf16* k;
  const bf16* v;
  int vs;
  bool there;
};
__device__ __forceinline__ TileAt prefix_tile(const AttnArgs& a, const Unit& u, int t) {
  return {a.kc + ((size_t)u.kh * a.cap + (size_t)t * kTileKeys) * a.Dh, a.vc + (size_t)u.kh * a.Dh * a.cap + (size_t)t * kTileKeys,
          a.cap, true};
}
__device__ __forceinline__ TileAt page_tile(const AttnArgs& a, const Unit& u, int id) {
  const bool there = id >= 0 && id < a.n_pages;  // (otherwise: any page, and none of its keys)
  const size_t at = ((size_t)(there ? id : 0) * a.Hkv + u.kh) * kPage * a.Dh;
  return {a.kp + at, a.vp + at, kPage, there};
}
// Page ids of a run, 64 at a time in the lanes of a wave.
struct PageIds {
  int ids, base;
  __device__ void start(const Unit& u, int t) {
    base = t;
    const int at = t + (int)(threadIdx.x & 63);
    ids = at < u.last ? ldg(u.table + at) : -1;
  }
  __device__ int get(const Unit& u, int t) {
    if (t - base >= kWave) start(u, t);
    return __builtin_amdgcn_readlane(ids, t - base);
  }
};

// Direct global -> LDS copy of 16 bytes per lane: lane l's land at lds + 16 l
// (lds the same in every lane).
__device__ __forceinline__ void dma16(const void* src, char* lds) {
  __builtin_amdgcn_global_load_lds((const LLMCAD_GLOBAL void*)src, (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// Which of the 8 keys from `key` on a row sees, by its mask (keys before held
// are tokens all rows of the request see).
__device__ __forceinline__ uint32_t seen8(const uint32_t (&anc)[4], int key, int held, int lim) {
  uint32_t vis = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int t = key + e - held;
    const uint32_t w = t < 32 ? anc[0] : t < 64 ? anc[1] : t < 96 ? anc[2] : anc[3];
    const bool sees = key + e < lim && (t < 0 || (t < LLMCAD_MAX_NODES && ((w >> (t & 31)) & 1u)));
    vis |= sees ? 1u << e : 0u;
  }
  return vis;
}

// Keys that some rows see and others do not: an Inf or NaN among their values
// would reach the others as 0 x Inf.  Such values are left out of the product
// O^T += V^T P^T, and a product of their indicators with the rows' sight tells
// which outputs they belong to.
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ bool nonfinite(const bf16x8& v) {
  const u16x8 x = __builtin_bit_cast(u16x8, v) & (uint16_t)0x7f80;
  bool any = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) any |= x[e] == 0x7f80;
  return any;
}
// v without its Inf and NaN; o with what they give the rows that see them.
__device__ __forceinline__ f32x4 take_nonfinite(bf16x8& v, uint32_t vis, f32x4 o) {
  constexpr uint16_t one = 0x3f80;  // (bf16 1)
  const u16x8 x = __builtin_bit_cast(u16x8, v);
  u16x8 up, down, sees, kept;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const bool bad = (x[e] & 0x7f80) == 0x7f80, nan = bad && (x[e] & 0x7f);
    up[e] = bad && (nan || !(x[e] & 0x8000)) ? one : (uint16_t)0;
    down[e] = bad && (nan || (x[e] & 0x8000)) ? one : (uint16_t)0;
    sees[e] = (vis >> e) & 1u ? one : (uint16_t)0;
    kept[e] = bad ? (uint16_t)0 : x[e];
  }
  v = __builtin_bit_cast(bf16x8, kept);
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const bf16x8 s = __builtin_bit_cast(bf16x8, sees);
  const f32x4 ups = mfma16x16x32(__builtin_bit_cast(bf16x8, up), s, zero);
  const f32x4 downs = mfma16x16x32(__builtin_bit_cast(bf16x8, down), s, zero);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (ups[i] > 0.0f) o[i] += INFINITY;
    if (downs[i] > 0.0f) o[i] -= INFINITY;
  }
  return o;
}

// ---------------------------------------------------------------- many rows
//
// 64 RB pairs per workgroup, 16 RB per wave.  Tiles of 64 keys are shared
// through LDS in fragment order (every access is 16 bytes per lane, lane by
// lane), keys and values in two buffers each.  A turn of the loop takes the
// values of tile t and the keys of tile t + 1: the scores of the next tile and
// the exponentials of this one need different units, and their instructions
// alternate.  Meanwhile the values of t + 1 and the keys of t + 2 are on their
// way to registers; they go to the buffers that this turn does not read, so one
// barrier per turn does.
//
// The running maximum is only a reference point: any value near it serves, so
// the output is rescaled only when some score exceeds it by 2^kSlack, and
// until then no lane needs another's scores.  The sums are per lane, joined at
// the end.  Probabilities (up to 2^kSlack) enter the value product in bf16, half
// a step of 2^-8 each.
template <int DH, int RB, bool PAGED>
struct TileWork {
  static constexpr int NS = Frags<DH>::NS, NB = Frags<DH>::NB;
  static constexpr int PER = 2 * NS;              // fragments a wave fetches per tile: K of a step, or V^T of a step
  static constexpr int HALF = 2 * PER * 1024;     // a tile's keys, or its values
  static_assert(2 * NS == NB, "as many key as value fragments");
  typedef f32x4 Scores[RB][4];  // [row block][step, key block]

  const AttnArgs& a;
  const Unit& u;
  char* lds;  // keys of even tiles, of odd tiles, values of even, of odd
  int lane, li, g, wave, group;
  bf16x8 qf[RB][NS];
  float m[RB], neg_m[RB], l[RB];
  f32x4 o[RB][NB];
  uint32_t vis[RB][2];
  bool masked, there;
  PageIds pages;
  uint32_t lane_k, lane_v;  // byte offsets of the lane's part of a tile's fragments

  __device__ __forceinline__ TileWork(const AttnArgs& a_, const Unit& u_, char* lds_) : a(a_), u(u_), lds(lds_) {
    lane = threadIdx.x & 63;
    li = lane & 15;
    g = lane >> 4;
    wave = wave_index();
    group = a.H / a.Hkv;
  }
  __device__ __forceinline__ int pair_of(int rb) const { return u.pair0 + (wave * RB + rb) * 16 + li; }
  __device__ __forceinline__ int clamped(int rb) const { return pair_of(rb) < u.pairs ? pair_of(rb) : u.pairs - 1; }
  // waves 0 and 2 fetch the keys of a tile's two steps, 1 and 3 the values
  __device__ __forceinline__ bool values() const { return (wave & 1) != 0; }
  __device__ __forceinline__ int key_of() const { return 32 * (wave >> 1); }

  // copies this wave's part of tile t straight to LDS
  __device__ __forceinline__ void fetch(int t) {
    const TileAt at = PAGED ? page_tile(a, u, pages.get(u, t)) : prefix_tile(a, u, t);
    char* to = lds + ((values() ? 2 : 0) + (t & 1)) * HALF + (wave >> 1) * PER * 1024;
    if (values()) {
#pragma unroll
      for (int e = 0; e < PER; ++e) dma16((const char*)(at.v + (size_t)e * 16 * at.vs) + lane_v, to + e * 1024);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e) dma16((const char*)(at.k + (e / NS) * 4 * DH + (e % NS) * 32) + lane_k, to + e * 1024);
    }
  }

  // scores of tile t (its keys in LDS)
  __device__ __forceinline__ void scores(Scores& sc, int t) {
    const char* at = lds + (t & 1) * HALF + lane * 16;
#pragma unroll
    for (int sb = 0; sb < 4; ++sb) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) sc[rb][sb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const bf16x8 k = lds_ld<bf16x8>(at + (sb * NS + s) * 1024);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) sc[rb][sb] = mfma16x16x32(k, qf[rb][s], sc[rb][sb]);
      }
    }
  }
  // the mask of tile t, and a new reference point where its scores need one
  __device__ __forceinline__ void look(Scores& sc, int t) {
    there = true;
    if (PAGED) {
      const int id = pages.get(u, t);
      there = id >= 0 && id < a.n_pages;
    }
    masked = (t + 1) * kTileKeys > u.held || !there;  // (not every row sees every key)
    if (masked) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        uint32_t anc[4] = {0, 0, 0, 0};
        if (PAGED) {
          const size_t row = (size_t)u.row0 + clamped(rb) / group;
#pragma unroll
          for (int j = 0; j < 4; ++j) anc[j] = ldg(a.mask + row * 4 + j);
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          vis[rb][st] = there ? seen8(anc, t * kTileKeys + 32 * st + 8 * g, u.held, u.lim) : 0u;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!((vis[rb][st] >> e) & 1u)) sc[rb][2 * st + (e >> 2)][e & 3] = -INFINITY;
        }
      }
    }
    float mx[RB];
    bool grow = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      mx[rb] = sc[rb][0][0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx[rb] = fmaxf(mx[rb], sc[rb][e >> 2][e & 3]);
      mx[rb] *= a.scale_log2;
      grow |= mx[rb] > m[rb] + kSlack;
    }
    if (__any(grow)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
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
  }
  __device__ __forceinline__ bf16x8 value(int t, int st, int db) const {
    return lds_ld<bf16x8>(lds + (2 + (t & 1)) * HALF + (st * NB + db) * 1024 + lane * 16);
  }
  // Values of keys that are not there count as zeros (what lies there may be NaN).
  __device__ __forceinline__ void clear_absent(int t) {
#pragma unroll 1
    for (int st = 0; st < 2; ++st) {
      const int valid = there ? u.lim - (t * kTileKeys + 32 * st + 8 * g) : 0;
      if (__any(valid < 8)) {
        char* at = lds + (2 + (t & 1)) * HALF + st * NB * 1024 + lane * 16;
#pragma unroll 1
        for (int db = wave; db < NB; db += kWaves) {
          bf16x8 v = lds_ld<bf16x8>(at + db * 1024);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (e >= valid) v[e] = (bf16)0.0f;
          lds_st<bf16x8>(at + db * 1024, v);
        }
      }
    }
    __syncthreads();
  }
  // Tile t's probabilities and its part of the output; the next tile's scores.
  __device__ __forceinline__ void turn(Scores& sc, Scores& next, int t) {
    const bool more = t + 1 < u.last;
    if (values() ? more : t + 2 < u.last) fetch(values() ? t + 1 : t + 2);
    bool bad = false;
    if (PAGED && masked) {
#pragma unroll
      for (int e = 0; e < 2 * NB; ++e) bad |= nonfinite(value(t, e / NB, e % NB));
    }
    scores(next, t + 1);  // (past the last tile: of what lies there, not used)
    bf16x8 p[RB][2];
#pragma unroll
    for (int st = 0; st < 2; ++st)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[rb][2 * st + (e >> 2)][e & 3], a.scale_log2, neg_m[rb]));
          l[rb] += v;
          p[rb][st][e] = f2bf(v);
        }
    if (PAGED && __any(bad)) {
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < NB; ++db) {
          const bf16x8 v = value(t, st, db);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            bf16x8 kept = v;
            o[rb][db] = take_nonfinite(kept, vis[rb][st], o[rb][db]);
            o[rb][db] = mfma16x16x32(kept, p[rb][st], o[rb][db]);
          }
          __builtin_amdgcn_sched_barrier(0);  // (one block's values at a time: the registers)
        }
    } else {
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int db = 0; db < NB; ++db) {
          const bf16x8 v = value(t, st, db);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) o[rb][db] = mfma16x16x32(v, p[rb][st], o[rb][db]);
        }
    }
    __syncthreads();
    if (more) {
      look(next, t + 1);
      if (masked && ((t + 2) * kTileKeys > u.lim || !there)) clear_absent(t + 1);
    }
  }

  __device__ __forceinline__ void run() {
    if (PAGED) pages.start(u, u.first);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m[rb] = -INFINITY;
      neg_m[rb] = 0.0f;
      l[rb] = 0.0f;
#pragma unroll
      for (int db = 0; db < NB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (u.first < u.last) {
      lane_k = ((key_of() + 8 * (li >> 2) + (li & 3)) * DH + 8 * g) * 2;
      lane_v = ((uint32_t)li * (PAGED ? kPage : a.cap) + key_of() + 8 * g) * 2;
      fetch(u.first);
      if (!values() && u.first + 1 < u.last) fetch(u.first + 1);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int pr = clamped(rb);
        const bf16* q = a.q + (size_t)(u.row0 + pr / group) * a.q_stride + (size_t)(u.kh * group + pr % group) * DH + 8 * g;
#pragma unroll
        for (int s = 0; s < NS; ++s) qf[rb][s] = ldg((const bf16x8*)(q + 32 * s));
      }
      __syncthreads();
      Scores A, B;
      scores(A, u.first);
      // (the first turn overwrites this tile's keys: every wave has read them)
      __syncthreads();
      look(A, u.first);
      if (masked && ((u.first + 1) * kTileKeys > u.lim || !there)) clear_absent(u.first);
      for (int t = u.first; t < u.last; t += 2) {
        turn(A, B, t);
        if (t + 1 < u.last) turn(B, A, t + 1);
      }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int pr = pair_of(rb);
      const float sum = col4_sum(l[rb]);
      if (pr >= u.pairs) continue;
      const size_t at = (u.part + pr / group) * a.H + u.kh * group + pr % group;
#pragma unroll
      for (int db = 0; db < NB; ++db) stg((f32x4*)(a.part_o + at * DH + 16 * db + 4 * g), o[rb][db]);
      if (g == 0) {
        stg(a.part_ml + at * 2, m[rb]);
        stg(a.part_ml + at * 2 + 1, sum);
      }
    }
  }
};

template <int DH, int RB, bool PAGED>
__device__ __forceinline__ void tile_unit(const AttnArgs& a, const Unit& u, char* lds) {
  TileWork<DH, RB, PAGED> w(a, u, lds);
  w.run();
}

// ---------------------------------------------------------------- few rows
//
// 16 pairs at a time: the waves take every fourth 32-key step each and meet in
// LDS.  What such a unit takes is the time of its loads, so a wave fetches a
// step while it computes another, and the probabilities enter the value
// product as two bf16 halves (about 16 bits): the matrix cores have the time.
template <int DH>
struct KeyStep {
  bf16x8 f[Frags<DH>::LOADS];
};

template <int DH>
__device__ __forceinline__ void load_step(KeyStep<DH>& R, const TileAt& at, int key) {
  const int lane = threadIdx.x & 63, li = lane & 15, g = lane >> 4;
  constexpr int NS = Frags<DH>::NS, NB = Frags<DH>::NB;
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int s = 0; s < NS; ++s)
      R.f[b * NS + s] = ldg((const bf16x8*)(at.k + (key + 8 * (li >> 2) + 4 * b + (li & 3)) * DH + 32 * s + 8 * g));
#pragma unroll
  for (int db = 0; db < NB; ++db) R.f[2 * NS + db] = ldg((const bf16x8*)(at.v + (size_t)(16 * db + li) * at.vs + key + 8 * g));
}

template <int DH>
__device__ __forceinline__ void narrow_unit(const AttnArgs& a, const Unit& u, int pair0, char* lds) {
  constexpr int NS = Frags<DH>::NS, NB = Frags<DH>::NB;
  float(*o_s)[16][DH + 4] = (float(*)[16][DH + 4])lds;
  float(*ml_s)[16][2] = (float(*)[16][2])(lds + sizeof(float) * kWaves * 16 * (DH + 4));
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, g = lane >> 4, wave = wave_index();
  const int group = a.H / a.Hkv;
  const int pr = pair0 + li < u.pairs ? pair0 + li : u.pairs - 1;
  const size_t row = (size_t)u.row0 + pr / group;
  const int j0 = 2 * u.first + wave, j1 = u.last * kTileKeys <= u.lim ? 2 * u.last : (u.lim + 31) / 32;
  PageIds pages;
  if (u.table) pages.start(u, u.first);
  KeyStep<DH> A, B;
  bool there_a = false, there_b = false;
  auto fetch = [&](KeyStep<DH>& R, bool& there, int j) {
    const TileAt at = u.table ? page_tile(a, u, pages.get(u, j >> 1)) : prefix_tile(a, u, j >> 1);
    there = at.there;
    load_step<DH>(R, at, 32 * (j & 1));
  };
  if (j0 < j1) fetch(A, there_a, j0);
  bf16x8 qf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s)
    qf[s] = ldg((const bf16x8*)(a.q + row * a.q_stride + (size_t)(u.kh * group + pr % group) * DH + 32 * s + 8 * g));
  uint32_t anc[4] = {0, 0, 0, 0};
  if (u.table)
#pragma unroll
    for (int j = 0; j < 4; ++j) anc[j] = ldg(a.mask + row * 4 + j);
  float m = -INFINITY, l = 0.0f;
  f32x4 o[NB];
#pragma unroll
  for (int db = 0; db < NB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto compute = [&](KeyStep<DH>& R, bool there, int j) {
    if (!there) return;
    f32x4 sc[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      sc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) sc[b] = mfma16x16x32(R.f[b * NS + s], qf[s], sc[b]);
    }
    const bool masked = 32 * (j + 1) > u.held;
    const uint32_t vis = masked ? seen8(anc, 32 * j + 8 * g, u.held, u.lim) : 0xffu;
    float sv[8], mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sv[e] = (vis >> e) & 1u ? sc[e >> 2][e & 3] * a.scale_log2 : -INFINITY;
      mx = fmaxf(mx, sv[e]);
    }
    if (__any(mx > m + kSlack)) {  // (the reference point moves)
      const float m_new = fmaxf(m, col4_max(mx));
      const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < NB; ++db) o[db] = o[db] * alpha;
    }
    const float m_use = m == -INFINITY ? 0.0f : m;
    bf16x8 ph, pl;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float p = __builtin_amdgcn_exp2f(sv[e] - m_use);
      l += p;
      ph[e] = f2bf(p);
      pl[e] = f2bf(p - bf2f(ph[e]));
    }
    bool bad = false;
    if (masked) {
      const int valid = u.lim - (32 * j + 8 * g);
#pragma unroll
      for (int db = 0; db < NB; ++db) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= valid) R.f[2 * NS + db][e] = (bf16)0.0f;
        bad |= nonfinite(R.f[2 * NS + db]);
      }
    }
    if (__any(bad))
#pragma unroll
      for (int db = 0; db < NB; ++db) {
        o[db] = take_nonfinite(R.f[2 * NS + db], vis, o[db]);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
    for (int db = 0; db < NB; ++db) {
      o[db] = mfma16x16x32(R.f[2 * NS + db], ph, o[db]);
      o[db] = mfma16x16x32(R.f[2 * NS + db], pl, o[db]);
    }
  };
  for (int j = j0; j < j1; j += 2 * kWaves) {
    if (j + kWaves < j1) fetch(B, there_b, j + kWaves);
    compute(A, there_a, j);
    if (j + 2 * kWaves < j1) fetch(A, there_a, j + 2 * kWaves);
    if (j + kWaves < j1) compute(B, there_b, j + kWaves);
  }
  // the four waves' states, joined in wave order
  l = col4_sum(l);
#pragma unroll
  for (int db = 0; db < NB; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) o_s[wave][li][16 * db + 4 * g + i] = o[db][i];
  if (g == 0) {
    ml_s[wave][li][0] = m;
    ml_s[wave][li][1] = l;
  }
  __syncthreads();
  for (int e = tid; e < 16 * DH; e += kThreads) {
    const int i = e / DH, c = e % DH, p = pair0 + i;
    if (p >= u.pairs) break;
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mm = fmaxf(mm, ml_s[w][i][0]);
    const float mu = mm == -INFINITY ? 0.0f : mm;
    float ll = 0.0f, oo = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(ml_s[w][i][0] - mu);
      ll += f * ml_s[w][i][1];
      oo += f * o_s[w][i][c];
    }
    const size_t at = (u.part + p / group) * a.H + u.kh * group + p % group;
    stg(a.part_o + at * DH + c, oo);
    if (c == 0) {
      stg(a.part_ml + at * 2, mm);
      stg(a.part_ml + at * 2 + 1, ll);
    }
  }
  __syncthreads();
}

// Unit x of the prefix: (K/V head, key split, row tile), row tiles fastest.
// Workgroup w runs on XCD w % 8: each XCD gets a contiguous share of the units, so
// that a (head, split)'s keys are read into one L2.
__device__ __forceinline__ bool prefix_unit(const AttnArgs& a, int w, int units, int row_tiles, Unit& u, int& tile) {
  const int share = up_div(units, 8), x = (w & 7) * share + (w >> 3);
  if ((w >> 3) >= share || x >= units) return false;
  const int split = x / row_tiles % a.KP, tiles = up_div(a.P, kTileKeys), per = up_div(tiles, a.KP);
  tile = x % row_tiles;
  u.kh = x / row_tiles / a.KP;
  u.row0 = 0;
  u.pairs = a.N * (a.H / a.Hkv);
  u.first = split * per < tiles ? split * per : tiles;
  u.last = u.first + per < tiles ? u.first + per : tiles;
  u.lim = u.held = a.P;
  u.table = nullptr;
  u.part = (size_t)split * a.N;
  u.pair0 = 0;
  return true;
}

template <int DH>
__global__ __launch_bounds__(kThreads, 2) void prefix_kernel(AttnArgs a, int units, int row_tiles) {
  __shared__ __align__(16) char lds[4 * Frags<DH>::LOADS * 1024];
  Unit u;
  int tile;
  if (!prefix_unit(a, blockIdx.x, units, row_tiles, u, tile)) return;
  u.pair0 = 128 * tile;
  tile_unit<DH, 2, false>(a, u, lds);
}

// Workgroups of few rows of the prefix first, then a.merge runs of a request's
// pages each.
template <int DH>
__global__ __launch_bounds__(kThreads, 2) void unit_kernel(AttnArgs a, int prefix_units, int row_tiles) {
  constexpr int kTileBytes = 4 * Frags<DH>::LOADS * 1024, kJoinBytes = kWaves * 16 * (DH + 6) * 4;
  __shared__ __align__(16) char lds[kTileBytes > kJoinBytes ? kTileBytes : kJoinBytes];
  const int group = a.H / a.Hkv;
  Unit u;
  const int padded = up_div(prefix_units, 8) * 8;
  if ((int)blockIdx.x < padded) {
    int tile;
    if (prefix_unit(a, blockIdx.x, prefix_units, row_tiles, u, tile)) narrow_unit<DH>(a, u, 16 * tile, lds);
    return;
  }
  const int x = blockIdx.x - padded, run_of = x / a.Hkv;
  u.kh = x % a.Hkv;
  if (run_of >= ldg(a.head + PLAN_UNITS)) return;
  const int unit = ldg(a.units + run_of), run = unit & 0xffff;
  const BatchRequest r = ldg(a.req + (unit >> 16));
  if (r.n == 0 || run % a.merge != 0) return;
  const int chunk = ldg(a.head + PLAN_CHUNK);
  u.row0 = r.row0;
  u.pairs = r.n * group;
  u.held = r.held;
  u.lim = r.held + r.n;
  u.table = a.table + (size_t)(unit >> 16) * a.max_pages;
  const int tiles = up_div(u.lim, kTileKeys) < a.max_pages ? up_div(u.lim, kTileKeys) : a.max_pages;
  const long long f = (long long)run * chunk, t = f + (long long)chunk * a.merge;
  u.first = f < tiles ? (int)f : tiles;
  u.last = t < tiles ? (int)t : tiles;
  u.part = (size_t)a.KP * a.N + r.part0 + (size_t)(run / a.merge) * r.n;
  u.pair0 = 0;
  if (u.pairs <= 16) {
    narrow_unit<DH>(a, u, 0, lds);
  } else {
    for (; u.pair0 < u.pairs; u.pair0 += 64) tile_unit<DH, 1, true>(a, u, lds);
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
  const int parts = a.KP + up_div(r.splits, a.merge);
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

// Few pairs of rows and heads per K/V head: the waves share 16 of them and split the keys; many:
// the waves split the pairs and share the keys.
bool wide_prefix(int N, int H, int Hkv) { return (long long)N * (H / Hkv) > 64; }

template <int DH>
hipError_t launch_attention(AttnArgs a, hipStream_t st) {
  const bool wide = wide_prefix(a.N, a.H, a.Hkv);
  // The plan cuts the requests' pages for 8 K/V heads; more heads make enough
  // workgroups of longer runs.
  a.merge = a.Hkv <= 8 ? 1 : cdiv(a.Hkv, 12);
  const int row_tiles = cdiv(a.N * (a.H / a.Hkv), wide ? 128 : 16);
  int units = row_tiles * a.KP * a.Hkv;
  const long long most = (long long)a.B * cdiv(a.max_pages, 2);  // (a run has two pages or more)
  const int runs = most < plan_max_units(a.B) ? (int)most : plan_max_units(a.B);
  if (wide && units > 0) {
    prefix_kernel<DH><<<dim3(cdiv(units, 8) * 8), dim3(kThreads), 0, st>>>(a, units, row_tiles);
    units = 0;
  }
  unit_kernel<DH><<<dim3(cdiv(units, 8) * 8 + runs * a.Hkv), dim3(kThreads), 0, st>>>(a, units, row_tiles);
  join_kernel<DH><<<dim3((unsigned)(((long long)a.N * a.H + kWaves - 1) / kWaves)), dim3(kThreads), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

int prefix_splits(int N, int H, int Hkv, int P) {
  if (P <= 0) return 0;
  const int pairs = N * (H / Hkv);
  const bool wide = wide_prefix(N, H, Hkv);
  int KP = wide ? 512 / (cdiv(pairs, 128) * Hkv) : cdiv(512, cdiv(pairs, 16) * Hkv);
  const int most = cdiv(P, 2 * kTileKeys);
  if (KP > most) KP = most;
  if (KP > max_prefix_splits(N)) KP = max_prefix_splits(N);
  return KP < 1 ? 1 : KP;
}

hipError_t launch_batch_attention(const AttnArgs& a, hipStream_t st) {
  return a.Dh == 128 ? launch_attention<128>(a, st) : launch_attention<64>(a, st);
}

}  // namespace llmcad
