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
//
// One token per request: bound by the reads of the pages and the prefix (128 tokens,
// 32 query heads on 8 K/V heads of 128, behind 8192 positions and up to 1024 tokens of
// their own: 83 us, 305 MB read, 3.6 TB/s; the narrow units' loads are 16 rows of
// 64 bytes, and a wave waits for all it has in flight twice a step).  Trees: bound by
// the instructions beside the matrix products (32 trees of 41, 40 heads of 128, behind
// 4099: 194 to 200 us, 650 to 700 TFLOP/s in the first launch, the matrix cores busy 41% of
// it, 491 MB read where each byte once is 463).
#include "batch.h"

namespace llmcad {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kWideRows = 128;  // pairs per workgroup of the prefix, where there are many
constexpr int kTileKeys = kPage;  // keys that units are cut by: a page
constexpr float kSlack = 8.0f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));

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
// Page ids of a run, 64 at a time in the lanes of a wave (and still those of the
// last few pages when the next 64 come).
struct PageIds {
  int ids, base;
  __device__ void start(const Unit& u, int t) {
    base = t;
    const int at = t + (int)(threadIdx.x & 63);
    ids = at < u.last ? ldg(u.table + at) : -1;
  }
  __device__ int get(const Unit& u, int t) {
    if (t - base >= kWave) start(u, t - 8);
    return __builtin_amdgcn_readlane(ids, t - base);
  }
};

// A row of the prefix's units that belongs to no placed request.  Its scores are all 0 around a
// reference point of 0: whatever lies in its query, it moves no other row's reference
// point (a wave moves those of its rows together).
__device__ __forceinline__ bool no_request(const AttnArgs& a, int row) { return ldg(a.row_req + row) < 0; }

// Direct global -> LDS copy of 16 bytes per lane: lane l's land at lds + 16 l
// (lds the same in every lane).
__device__ __forceinline__ void dma16(const void* src, char* lds) {
  __builtin_amdgcn_global_load_lds((const LLMCAD_GLOBAL void*)src, (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// Which of the 8 keys from `key` on a row sees, by its mask: all before held,
// those that the mask names from there on, none from lim on.
__device__ __forceinline__ uint32_t seen8(const uint32_t (&anc)[4], int key, int held, int lim) {
  const int off = key - held;  // (keys of the request's rows: bits off .. off + 7 of the mask)
  const int at = off < 0 ? 0 : off;
  const uint32_t lo = at < 32 ? anc[0] : at < 64 ? anc[1] : at < 96 ? anc[2] : anc[3];
  const uint32_t hi = at < 32 ? anc[1] : at < 64 ? anc[2] : at < 96 ? anc[3] : 0u;
  uint32_t vis = at < LLMCAD_MAX_NODES ? (uint32_t)((((uint64_t)hi << 32) | lo) >> (at & 31)) : 0u;
  const int before = -off < 0 ? 0 : -off > 8 ? 8 : -off;  // (held tokens among the eight)
  vis = vis << before | ((1u << before) - 1u);
  const int there = lim - key < 0 ? 0 : lim - key > 8 ? 8 : lim - key;
  return vis & ((1u << there) - 1u);
}
// The 8 values of a fragment whose keys are there (bits of `there`; the others
// count as zeros: what lies in them may be NaN): masks for its four words.
__device__ __forceinline__ u32x4 kept_words(uint32_t there) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = ((there >> (2 * i)) & 1u ? 0xffffu : 0u) | ((there >> (2 * i + 1)) & 1u ? 0xffff0000u : 0u);
  return w;
}
__device__ __forceinline__ bf16x8 keep(bf16x8 v, u32x4 words) {
  return __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, v) & words);
}

// Keys that some rows see and others do not: an Inf or NaN among their values
// would reach the others as 0 x Inf.  Such values are left out of the product
// O^T += V^T P^T, and a product of their indicators with the rows' sight tells
// which outputs they belong to; those get them at the end.
// The largest magnitudes of the values seen so far, two by two.
__device__ __forceinline__ void largest(u16x8& most, const bf16x8& v) {
  most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x8, v) & (uint16_t)0x7fff);
}
__device__ __forceinline__ bool nonfinite(const u16x8& most) {
  bool any = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) any |= most[e] >= 0x7f80;
  return any;
}
// What the Inf and NaN of a fragment give the outputs of the rows that see them:
// bit 4 db + i of up (+Inf), of down (-Inf); both: NaN.
struct Strays {
  uint32_t up = 0, down = 0;
  __device__ __forceinline__ void note(const bf16x8& v, uint32_t vis, int db) {
    constexpr uint16_t one = 0x3f80;  // (bf16 1)
    const u16x8 x = __builtin_bit_cast(u16x8, v);
    u16x8 ups, downs, sees;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool bad = (x[e] & 0x7f80) == 0x7f80, nan = bad && (x[e] & 0x7f);
      ups[e] = bad && (nan || !(x[e] & 0x8000)) ? one : (uint16_t)0;
      downs[e] = bad && (nan || (x[e] & 0x8000)) ? one : (uint16_t)0;
      sees[e] = (vis >> e) & 1u ? one : (uint16_t)0;
    }
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const bf16x8 s = __builtin_bit_cast(bf16x8, sees);
    const f32x4 a = mfma16x16x32(__builtin_bit_cast(bf16x8, ups), s, zero);
    const f32x4 b = mfma16x16x32(__builtin_bit_cast(bf16x8, downs), s, zero);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      up |= a[i] > 0.0f ? 1u << (4 * db + i) : 0u;
      down |= b[i] > 0.0f ? 1u << (4 * db + i) : 0u;
    }
  }
  template <int NB>
  __device__ __forceinline__ void give(f32x4 (&o)[NB]) const {
    if (!__any((up | down) != 0u)) return;
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((up >> (4 * db + i)) & 1u) o[db][i] += INFINITY;
        if ((down >> (4 * db + i)) & 1u) o[db][i] -= INFINITY;
      }
  }
};
__device__ __forceinline__ bf16x8 finite(const bf16x8& v) {
  u16x8 x = __builtin_bit_cast(u16x8, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (x[e] & 0x7f80) == 0x7f80 ? (uint16_t)0 : x[e];
  return __builtin_bit_cast(bf16x8, x);
}

// ---------------------------------------------------------------- many rows
//
// 64 RB pairs per workgroup, 16 RB per wave.  Tiles of 32 keys are shared
// through LDS, in two buffers: while one is computed the next is copied.  (So in
// the prefix.  In pages look() asks for the tile's page again, a lane of a register
// that may have just been loaded, and waits there for the next tile's copy too: it
// overlaps the score products alone.)
//
// Two row blocks per wave for the prefix: each fragment read from LDS feeds two
// products, in 168 registers, three waves per SIMD (three or four blocks leave one
// wave, and nothing runs beside it: slower).  64-key tiles with two waves per SIMD
// read the prefix 7% faster and the mix of prefix and pages slower.
//
// The running maximum is only a reference point: any value near it serves, so
// the output is rescaled only when some score exceeds it by 2^kSlack, and
// until then no lane needs another's scores.  The sums are per lane, joined at
// the end.  Probabilities (up to 2^kSlack) enter the value product in bf16, half
// a step of 2^-8 each: 0.0023 of the outputs against 64 bits, where their own rounding
// is 0.0017.  (Two bf16 parts, as with few rows, were measured: 16 trees of 31 rows 46 us
// and 55, 32 of 41 194 and 244, 128 tokens 84 and 86; the matrix products are the price.)
template <int DH, int RB, bool PAGED>
struct TileWork {
  static constexpr int NS = Frags<DH>::NS, NB = Frags<DH>::NB;
  static constexpr int KEYS = 32;               // of a tile: half a page
  static constexpr int PARTS = kTileKeys / KEYS;
  static constexpr int HALF = KEYS * DH * 2;    // bytes of a tile's keys, or of its values
  static constexpr int FLAG = 4 * HALF;         // (a flag behind the buffers)
  static constexpr int LDS = FLAG + 16;
  static constexpr int PER = HALF / 2048;       // KiB that a wave fetches: half of the keys, or of the values
  typedef f32x4 Scores[RB][2];                  // [row block][key block]

  const AttnArgs& a;
  const Unit& u;
  char* lds;  // keys of even tiles, of odd tiles, values of even, of odd
  int first, last;  // tiles
  int lane, li, g, wave, group;
  bf16x8 qf[RB][NS];
  float m[RB], neg_m[RB], l[RB];
  f32x4 o[RB][NB];
  Strays strays[RB];
  bool there;
  PageIds pages;
  const char* src;          // where this wave's part of the next tile to fetch begins
  uint32_t lane_at[PER];    // byte offsets from there of the lane's pieces, by KiB

  __device__ __forceinline__ TileWork(const AttnArgs& a_, const Unit& u_, char* lds_) : a(a_), u(u_), lds(lds_) {
    lane = threadIdx.x & 63;
    li = lane & 15;
    g = lane >> 4;
    wave = wave_index();
    group = a.H / a.Hkv;
    first = u.first * PARTS;
    const int end = (u.lim + KEYS - 1) / KEYS;
    last = u.last * PARTS < end ? u.last * PARTS : end;
  }
  __device__ __forceinline__ int pair_of(int rb) const { return u.pair0 + (wave * RB + rb) * 16 + li; }
  __device__ __forceinline__ int clamped(int rb) const { return pair_of(rb) < u.pairs ? pair_of(rb) : u.pairs - 1; }

  // LDS holds a tile's keys as [key block][16 rows][DH] and its values as
  // [DH][KEYS], so that a KiB copied to it is whole rows: 64 lanes read 4 to 16
  // rows of 64 to 256 contiguous bytes.  (In fragment order each lane's 16 bytes
  // are another row than its neighbours', and the vector cache takes them one by
  // one: 67 accesses per KiB instead of 19.)  The 16-byte pieces of a row are swapped by its
  // index, so that the pieces of 16 rows that a fragment reads together lie in
  // different banks (a read takes 256 bytes of LDS at a time).
  static constexpr int ROW = DH * 2, VROW = KEYS * 2;  // bytes of a row of keys, of values
  static constexpr int ROWS = 1024 / ROW, DIMS = 1024 / VROW;  // of them in a KiB
  __device__ static __forceinline__ int swap(int row_bytes, int row) {
    return row_bytes == 256 ? row & 15 : row_bytes == 128 ? (row >> 1) & 7 : (row >> 2) & 3;
  }
  __device__ __forceinline__ const char* key_at(int t, int sb, int s) const {
    return lds + (t & 1) * HALF + sb * 16 * ROW + li * ROW + (((4 * s + g) ^ swap(ROW, li)) * 16);
  }
  __device__ __forceinline__ char* value_at(int t, int db) const {
    return lds + (2 + (t & 1)) * HALF + (16 * db + li) * VROW + ((g ^ swap(VROW, li)) * 16);
  }
  // waves 0 and 1 fetch a key block each, 2 and 3 half of the values' dims each
  __device__ __forceinline__ bool values() const { return wave >= 2; }
  __device__ __forceinline__ void place_lanes() {
    const int part = wave & 1;
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (values()) {  // dims DIMS (PER part + e) ..
        const int dim = DIMS * (PER * part + e) + lane / (VROW / 16), piece = lane % (VROW / 16);
        lane_at[e] = ((uint32_t)dim * (PAGED ? kPage : a.cap) + 8 * (piece ^ swap(VROW, dim & 15))) * 2;
      } else {  // key block `part`, rows ROWS e .. of it (key 8 (row / 4) + 4 part + row % 4)
        const int row = ROWS * e + lane / (ROW / 16), piece = lane % (ROW / 16);
        lane_at[e] = (8 * (row >> 2) + 4 * part + (row & 3)) * ROW + (piece ^ swap(ROW, row)) * 16;
      }
    if (!PAGED) set_src(prefix_tile(a, u, first / PARTS), first);
  }
  __device__ __forceinline__ void set_src(const TileAt& at, int t) {
    const int key = t % PARTS * KEYS;
    src = values() ? (const char*)(at.v + key) : (const char*)(at.k + key * DH);
  }
  // copies this wave's part of tile t straight to LDS (called for one tile after the other)
  __device__ __forceinline__ void fetch(int t) {
    if (PAGED && (t % PARTS == 0 || t == first)) set_src(page_tile(a, u, pages.get(u, t / PARTS)), t);
    char* to = lds + ((values() ? 2 : 0) + (t & 1)) * HALF + (wave & 1) * PER * 1024;
#pragma unroll
    for (int e = 0; e < PER; ++e) dma16(src + lane_at[e], to + e * 1024);
    src += values() ? VROW : KEYS * ROW;
  }

  // scores of tile t (its keys in LDS)
  __device__ __forceinline__ void scores(Scores& sc, int t) {
#pragma unroll
    for (int sb = 0; sb < 2; ++sb) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) sc[rb][sb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const bf16x8 k = lds_ld<bf16x8>(key_at(t, sb, s));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) sc[rb][sb] = mfma16x16x32(k, qf[rb][s], sc[rb][sb]);
      }
    }
  }
  // Clears, where they lie, tile t's values of keys that are not there, and takes
  // out the Inf and NaN of those that some rows see and others do not.  A wave does
  // a quarter; all waves of the workgroup come here for the same tiles.
  __device__ __forceinline__ void clean(int t, const uint32_t (&vis)[RB]) {
    int* flag = (int*)(lds + FLAG);
    u16x8 most = (uint16_t)0;
#pragma unroll 1
    for (int db = wave; db < NB; db += kWaves) {
      char* at = value_at(t, db);
      const int left = u.lim - (t * KEYS + 8 * g);
      const bf16x8 v = keep(lds_ld<bf16x8>(at), kept_words(!there || left <= 0 ? 0u : left >= 8 ? 0xffu : (1u << left) - 1u));
      if (PAGED) largest(most, v);
      lds_st<bf16x8>(at, v);
    }
    if (PAGED && __any(nonfinite(most)) && lane == 0) *flag = 1;
    __syncthreads();
    if (PAGED && *flag != 0) {
#pragma unroll 1
      for (int db = 0; db < NB; ++db) {
        const bf16x8 v = lds_ld<bf16x8>(value_at(t, db));
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) strays[rb].note(v, vis[rb], db);
      }
      __syncthreads();
      if (threadIdx.x == 0) *flag = 0;
#pragma unroll 1
      for (int db = wave; db < NB; db += kWaves) {
        char* at = value_at(t, db);
        lds_st<bf16x8>(at, finite(lds_ld<bf16x8>(at)));
      }
      __syncthreads();
    }
  }
  // The mask of tile t, and a new reference point where its scores need one.
  __device__ __forceinline__ void look(Scores& sc, int t) {
    there = true;
    if (PAGED) {
      const int id = pages.get(u, t / PARTS);
      there = id >= 0 && id < a.n_pages;
    }
    if ((t + 1) * KEYS > u.held || !there) {  // (not every row sees every key)
      uint32_t vis[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        uint32_t anc[4] = {0, 0, 0, 0};
        if (PAGED) {
          const size_t row = (size_t)u.row0 + clamped(rb) / group;
#pragma unroll
          for (int j = 0; j < 4; ++j) anc[j] = ldg(a.mask + row * 4 + j);
        }
        vis[rb] = there ? seen8(anc, t * KEYS + 8 * g, u.held, u.lim) : 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!((vis[rb] >> e) & 1u)) sc[rb][e >> 2][e & 3] = -INFINITY;
      }
      clean(t, vis);
    }
    float mx[RB];
    bool grow = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      mx[rb] = sc[rb][0][0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx[rb] = fmaxf(mx[rb], sc[rb][e >> 2][e & 3]);
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
  // Tile t's probabilities and its part of the output.
  __device__ __forceinline__ void add(Scores& sc, int t) {
    bf16x8 p[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[rb][e >> 2][e & 3], a.scale_log2, neg_m[rb]));
        l[rb] += v;
        p[rb][e] = f2bf(v);
      }
#pragma unroll
    for (int db = 0; db < NB; ++db) {
      const bf16x8 v = lds_ld<bf16x8>(value_at(t, db));
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) o[rb][db] = mfma16x16x32(v, p[rb], o[rb][db]);
    }
  }
  __device__ __forceinline__ void run() {
    if (PAGED) pages.start(u, u.first);
    place_lanes();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      m[rb] = -INFINITY;
      neg_m[rb] = 0.0f;
      l[rb] = 0.0f;
#pragma unroll
      for (int db = 0; db < NB; ++db) o[rb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (threadIdx.x == 0) *(int*)(lds + FLAG) = 0;
    if (first < last) {
      fetch(first);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int pr = clamped(rb);
        const bool nobody = !PAGED && no_request(a, u.row0 + pr / group);
        const bf16* q = a.q + (size_t)(u.row0 + pr / group) * a.q_stride + (size_t)(u.kh * group + pr % group) * DH + 8 * g;
#pragma unroll
        for (int s = 0; s < NS; ++s) qf[rb][s] = ldg((const bf16x8*)(q + 32 * s));
        if (nobody) {
          m[rb] = 0.0f;
#pragma unroll
          for (int s = 0; s < NS; ++s) qf[rb][s] = (bf16)0.0f;
        }
      }
      __syncthreads();
      for (int t = first; t < last; ++t) {
        Scores sc;
        if (t + 1 < last) fetch(t + 1);
        scores(sc, t);
        look(sc, t);
        add(sc, t);
        __syncthreads();
      }
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int pr = pair_of(rb);
      const float sum = col4_sum(l[rb]);
      if (PAGED) strays[rb].give(o[rb]);
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

// ---------------------------------------------------------------- few rows
//
// 16 pairs at a time: the waves take every fourth 32-key step each and meet in
// LDS.  What such a unit takes is the time of its loads.  A wave issues the next
// step's keys as soon as the scores have taken this one's, and its values behind
// the value product, but does not overlap them with its own work: the score products wait
// for everything (the queries are the youngest loads in front of the loop), and so
// does the next step's page, whose lane may have just been loaded; other
// workgroups fill the time.  The probabilities enter the value product as two
// bf16 halves (about 16 bits): the matrix cores have the time.
template <int DH>
__device__ __forceinline__ void narrow_unit(const AttnArgs& a, const Unit& u, char* lds) {
  constexpr int NS = Frags<DH>::NS, NB = Frags<DH>::NB;
  float(*o_s)[16][DH + 4] = (float(*)[16][DH + 4])lds;
  float(*ml_s)[16][2] = (float(*)[16][2])(lds + sizeof(float) * kWaves * 16 * (DH + 4));
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, g = lane >> 4, wave = wave_index();
  const int group = a.H / a.Hkv, pair0 = u.pair0;
  const int pr = pair0 + li < u.pairs ? pair0 + li : u.pairs - 1;
  const size_t row = (size_t)u.row0 + pr / group;
  const bool nobody = !u.table && no_request(a, (int)row);
  const int j0 = 2 * u.first + wave, j1 = u.last * kTileKeys <= u.lim ? 2 * u.last : (u.lim + 31) / 32;
  PageIds pages;
  if (u.table) pages.start(u, u.first);
  bf16x8 k[2 * NS], v[NB];
  const uint32_t lane_k = ((8 * (li >> 2) + (li & 3)) * DH + 8 * g) * 2;
  const uint32_t lane_v = ((uint32_t)li * (u.table ? kPage : a.cap) + 8 * g) * 2;
  auto where = [&](int j) { return u.table ? page_tile(a, u, pages.get(u, j >> 1)) : prefix_tile(a, u, j >> 1); };
  auto fetch_keys = [&](const TileAt& at, int j) {
    const bf16* src = at.k + 32 * (j & 1) * DH;
#pragma unroll
    for (int e = 0; e < 2 * NS; ++e) k[e] = ldg((const bf16x8*)((const char*)(src + (e / NS) * 4 * DH + (e % NS) * 32) + lane_k));
  };
  auto fetch_values = [&](const TileAt& at, int j) {
    const bf16* src = at.v + 32 * (j & 1);
#pragma unroll
    for (int db = 0; db < NB; ++db) v[db] = ldg((const bf16x8*)((const char*)(src + (size_t)(16 * db) * at.vs) + lane_v));
  };
  TileAt at = {nullptr, nullptr, 0, false};
  if (j0 < j1) {
    at = where(j0);
    fetch_keys(at, j0);
    fetch_values(at, j0);
  }
  bf16x8 qf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s)
    qf[s] = ldg((const bf16x8*)(a.q + row * a.q_stride + (size_t)(u.kh * group + pr % group) * DH + 32 * s + 8 * g));
  float m = nobody ? 0.0f : -INFINITY, l = 0.0f;
  if (nobody)
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = (bf16)0.0f;
  Strays strays;
  f32x4 o[NB];
#pragma unroll
  for (int db = 0; db < NB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int j = j0; j < j1; j += kWaves) {
    f32x4 sc[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      sc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < NS; ++s) sc[b] = mfma16x16x32(k[b * NS + s], qf[s], sc[b]);
    }
    const bool there = at.there, more = j + kWaves < j1;
    if (more) {
      at = where(j + kWaves);
      fetch_keys(at, j + kWaves);
    }
    const bool masked = 32 * (j + 1) > u.held || !there;
    uint32_t vis = 0xffu;
    if (masked) {
      uint32_t anc[4] = {0, 0, 0, 0};
      if (u.table)
#pragma unroll
        for (int w = 0; w < 4; ++w) anc[w] = ldg(a.mask + row * 4 + w);
      vis = there ? seen8(anc, 32 * j + 8 * g, u.held, u.lim) : 0u;
    }
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
    if (masked) {
      const int left = u.lim - (32 * j + 8 * g);
      const u32x4 words = kept_words(!there || left <= 0 ? 0u : left >= 8 ? 0xffu : (1u << left) - 1u);
      u16x8 most = (uint16_t)0;
#pragma unroll
      for (int db = 0; db < NB; ++db) {
        v[db] = keep(v[db], words);
        largest(most, v[db]);
      }
      if (__any(nonfinite(most))) {  // (through the wave's part of LDS: a short loop)
        char* mine = lds + wave * 16 * (DH + 4) * 4 + lane * 16;
        static_assert(NB * 1024 <= 16 * (DH + 4) * 4, "the values of a step in a wave's part");
#pragma unroll
        for (int db = 0; db < NB; ++db) lds_st<bf16x8>(mine + db * 1024, v[db]);
#pragma unroll 1
        for (int db = 0; db < NB; ++db) {
          const bf16x8 x = lds_ld<bf16x8>(mine + db * 1024);
          strays.note(x, vis, db);
          lds_st<bf16x8>(mine + db * 1024, finite(x));
        }
#pragma unroll
        for (int db = 0; db < NB; ++db) v[db] = lds_ld<bf16x8>(mine + db * 1024);
      }
    }
#pragma unroll
    for (int db = 0; db < NB; ++db) {
      o[db] = mfma16x16x32(v[db], ph, o[db]);
      o[db] = mfma16x16x32(v[db], pl, o[db]);
    }
    if (more) fetch_values(at, j + kWaves);
  }
  // A probability's second half may be 0 or negative, so that its product with an
  // Inf that every row sees is not that Inf: such outputs are set from the values.
  bool bad = false;
#pragma unroll
  for (int db = 0; db < NB; ++db)
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= !__builtin_isfinite(o[db][i]);
  if (__any(bad)) {
    Strays seen;
    if (u.table) pages.start(u, u.first);
#pragma unroll 1
    for (int j = j0; j < j1; j += kWaves) {
      at = where(j);
      if (32 * (j + 1) > u.held || !at.there) continue;  // (taken care of above)
#pragma unroll 1
      for (int db = 0; db < NB; ++db) {
        const bf16* src = at.v + 32 * (j & 1) + (size_t)(16 * db) * at.vs;
        seen.note(ldg((const bf16x8*)((const char*)src + lane_v)), 0xffu, db);
      }
    }
#pragma unroll
    for (int db = 0; db < NB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (((seen.up | seen.down) >> (4 * db + i)) & 1u) o[db][i] = 0.0f;
    strays.up |= seen.up;
    strays.down |= seen.down;
  }
  // the four waves' states, joined in wave order
  l = col4_sum(l);
  strays.give(o);
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

// The plan is for this call.  (A narrower table than the plan's gives fewer
// workgroups than the plan has runs.)
__device__ __forceinline__ bool plan_fits(const AttnArgs& a) {
  return plan_is_for(a.head, a.B, a.N) && ldg(a.head + PLAN_MAX_PAGES) <= a.max_pages;
}

// Workgroup x of the runs' part: a.merge runs of a request's pages for one K/V head.
__device__ __forceinline__ bool run_unit(const AttnArgs& a, int x, Unit& u) {
  const int run_of = x / a.Hkv;
  u.kh = x % a.Hkv;
  const BatchUnit r = ldg(a.units + run_of);  // (what lies behind the last one is not used)
  if (run_of >= ldg(a.head + PLAN_UNITS) || !plan_fits(a) || r.n == 0 || r.run % a.merge != 0) return false;
  u.row0 = r.row0;
  u.pairs = r.n * (a.H / a.Hkv);
  u.held = r.held;
  u.lim = r.held + r.n;
  u.table = a.table + (size_t)r.request * a.max_pages;
  const int tiles = up_div(u.lim, kTileKeys) < a.max_pages ? up_div(u.lim, kTileKeys) : a.max_pages;
  const long long f = (long long)r.run * r.chunk, t = f + (long long)r.chunk * a.merge;
  u.first = f < tiles ? (int)f : tiles;
  u.last = t < tiles ? (int)t : tiles;
  u.part = (size_t)a.KP * a.N + r.part0 + (size_t)(r.run / a.merge) * r.n;
  u.pair0 = 0;
  return true;
}

// The prefix's workgroups first (they are the longest), then those of the runs:
// three on a CU, so that the ones that wait for memory and the ones that
// compute share it.
template <int DH>
__global__ __launch_bounds__(kThreads, 3) void unit_kernel(AttnArgs a, int prefix_units, int row_tiles, int wide) {
  typedef TileWork<DH, 2, false> Prefix;
  typedef TileWork<DH, 1, true> Pages;
  constexpr int kJoin = kWaves * 16 * (DH + 6) * 4, kTile = Prefix::LDS > Pages::LDS ? Prefix::LDS : Pages::LDS;
  __shared__ __align__(16) char lds[kTile > kJoin ? kTile : kJoin];
  Unit u;
  const int padded = up_div(prefix_units, 8) * 8;
  bool few;
  if ((int)blockIdx.x < padded) {
    int tile;
    if (!prefix_unit(a, blockIdx.x, prefix_units, row_tiles, u, tile)) return;
    if (wide) {
      u.pair0 = kWideRows * tile;
      Prefix(a, u, lds).run();
      return;
    }
    u.pair0 = 16 * tile;
    u.pairs = u.pair0 + 16 < u.pairs ? u.pair0 + 16 : u.pairs;
    few = true;
  } else {
    if (!run_unit(a, blockIdx.x - padded, u)) return;
    few = u.pairs <= 16;
  }
  if (few)
    narrow_unit<DH>(a, u, lds);
  else
    for (; u.pair0 < u.pairs; u.pair0 += 64) Pages(a, u, lds).run();
}

// A row's partial results of a head, in the order of their keys: DH / 4 lanes with
// four dims each.  Each lane first takes one part's maximum and sum, so that the
// reads of the outputs wait for nothing but each other.  Bound by the parts' bytes
// (32 trees of 41 rows, 40 heads: 19 us, 55 MB of parts, 13 MB of results; 22.6 a
// wave per head with one part after the other).
template <int DH>
__global__ __launch_bounds__(kThreads) void join_kernel(AttnArgs a) {
  constexpr int LANES = DH / 4;
  const size_t item = ((size_t)blockIdx.x * kThreads + threadIdx.x) / LANES;
  const int lane = threadIdx.x % LANES;
  if (item >= (size_t)a.N * a.H) return;
  const int row = (int)(item / a.H), h = (int)(item % a.H);
  const int b = ldg(a.row_req + row);
  if (!plan_fits(a) || b < 0) return;  // (no request's row: left as it was)
  const BatchRequest r = ldg(a.req + b);
  const int parts = a.KP + up_div(r.splits, a.merge);
  auto place = [&](int p) {
    const size_t pr = p < a.KP ? (size_t)p * a.N + row
                               : (size_t)a.KP * a.N + r.part0 + (size_t)(p - a.KP) * r.n + (row - r.row0);
    return pr * a.H + h;
  };
  float m = -INFINITY, l = 0.0f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < parts; p0 += LANES) {
    float pm = -INFINITY, pl = 0.0f;
    if (p0 + lane < parts) {
      const float2 ml = ldg((const float2*)a.part_ml + place(p0 + lane));
      pm = ml.x;
      pl = ml.y;
    }
    float mm = pm;
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) mm = fmaxf(mm, __shfl_xor(mm, off, LANES));
    mm = fmaxf(mm, m);
    const float mu = mm == -INFINITY ? 0.0f : mm, fa = __builtin_amdgcn_exp2f(m - mu), f = __builtin_amdgcn_exp2f(pm - mu);
    pl *= f;
#pragma unroll
    for (int off = LANES / 2; off >= 1; off >>= 1) pl += __shfl_xor(pl, off, LANES);
    l = fa * l + pl;
    o = o * fa;
    m = mm;
    const int n = parts - p0 < LANES ? parts - p0 : LANES;
    for (int q = 0; q < n; q += 4) {
      f32x4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = q + i < n ? ldg((const f32x4*)(a.part_o + place(p0 + q + i) * DH) + lane) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) o += x[i] * __shfl(f, q + i, LANES);  // (f is 0 past the last part)
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  bf16x4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = f2bf(o[i] * inv);
  stg((bf16x4*)(a.out + item * DH) + lane, out);
}

// Few pairs of rows and heads per K/V head: the waves share 16 of them and split
// the keys; many: the waves split the pairs and share the keys through LDS.  (us,
// 32 heads of 128, narrow / wide: 41 rows behind 2048 positions 30.0 / 20.9, 64 rows
// behind 512 18.4 / 16.0 and behind 4096 40.9 / 28.0; up to 32 pairs the narrow ones
// win or tie: 16 rows behind 512 15.0 / 15.9, 31 behind 2048 19.7 / 19.8.)
bool wide_prefix(int N, int H, int Hkv) { return (long long)N * (H / Hkv) > 32; }

template <int DH>
hipError_t launch_attention(AttnArgs a, hipStream_t st) {
  const bool wide = wide_prefix(a.N, a.H, a.Hkv);
  // The plan cuts the requests' pages for 8 K/V heads; more heads make enough
  // workgroups of longer runs (us with runs joined for every 16 heads / for every
  // 12: one token after 4000 held ones 27.6 / 29.9, 60 tokens of 32 heads 118 / 122;
  // no difference elsewhere).
  a.merge = a.Hkv <= 8 ? 1 : cdiv(a.Hkv, 16);
  const int row_tiles = cdiv(a.N * (a.H / a.Hkv), wide ? kWideRows : 16);
  const int units = row_tiles * a.KP * a.Hkv;
  const long long most = (long long)a.B * cdiv(a.max_pages, 2);  // (a run has two pages or more)
  const int runs = (most < plan_max_units(a.B) ? (int)most : plan_max_units(a.B)) * a.Hkv;
  unit_kernel<DH><<<dim3(cdiv(units, 8) * 8 + runs), dim3(kThreads), 0, st>>>(a, units, row_tiles, wide);
  join_kernel<DH><<<dim3((unsigned)(((long long)a.N * a.H * (DH / 4) + kThreads - 1) / kThreads)), dim3(kThreads), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

// The prefix's workgroups, one per CU: they share the CUs with the runs', and
// every split leaves partial results.  (us with 128, 192, 256, 384 and 512 of them: 16
// trees of 31 rows, 32 heads, behind 2048 positions 69, 70, 49, 56, 60; 128 tokens, 8
// K/V heads, behind 8192 110, 97, 86, 94, 98; 16 tokens 33, 34, 35, 42, 51.  Narrow
// units, 128, 256 and 512: one token, 32 heads, behind 8192 43, 31, 33, 31 rows
// behind 2048 25, 20, 23.)
int prefix_splits(int N, int H, int Hkv, int P) {
  if (P <= 0) return 0;
  const int pairs = N * (H / Hkv);
  const bool wide = wide_prefix(N, H, Hkv);
  int KP = wide ? 256 / (cdiv(pairs, kWideRows) * Hkv) : cdiv(256, cdiv(pairs, 16) * Hkv);
  const int most = cdiv(P, 2 * kTileKeys);
  if (KP > most) KP = most;
  if (KP > max_prefix_splits(N)) KP = max_prefix_splits(N);
  return KP < 1 ? 1 : KP;
}

hipError_t launch_batch_attention(const AttnArgs& a, hipStream_t st) {
  return a.Dh == 128 ? launch_attention<128>(a, st) : launch_attention<64>(a, st);
}

}  // namespace llmcad
