// Operators for several requests behind one shared prefix: the layout of a
// step's plan and the launchers of their kernels (batch.hip, batch_attn.hip,
// scores.hip; host checks in batch_api.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "device.h"
#include "layout.h"
#include "llmcad.h"

namespace llmcad {

constexpr int kPage = LLMCAD_PAGE;                // slots of a page
constexpr int kMaxRequests = LLMCAD_MAX_REQUESTS;
// Key splits of the requests' own pages: a request's pages are cut into runs
// of one length, chosen so that there are about this many runs in all (one run
// per (K/V head, run) is a workgroup; 128 tokens of 8 K/V heads after up to 1024
// tokens each take 69 us with 96 runs, 64 with 192 and with 256) ...
constexpr int kSplitRuns = 192;
// ... and so that the rows' partial results stay below n_rows + max(n_rows, this).
constexpr int kSplitRows = 2048;

// Keeps the HIP status that llmcad_status_string reports for LLMCAD_EHIP (api.hip).
void keep_hip_error(hipError_t e);

// What the attention needs of one request, written by the plan kernel.
struct BatchRequest {
  int row0;    // first row
  int n;       // rows (0: the request sits the step out, or could not be placed)
  int held;    // tokens in its pages before the step
  int splits;  // runs of its pages
  int part0;   // its partial results: row i of run s is partial row part0 + s n + i
  int pad[3];
};

// A run of a request's pages, with all that a workgroup needs to begin on it.
struct BatchUnit {
  int request, run;
  int row0, n, held, part0;  // the request's
  int chunk;                 // pages per run
  int pad;
};

// Head of a plan (int32 words).
enum PlanWord { PLAN_UNITS = 0, PLAN_TAKEN = 1, PLAN_REQUESTS = 2, PLAN_ROWS = 3, PLAN_MAX_PAGES = 4, PLAN_WORDS = 64 };
// A plan for other sizes lies elsewhere in its buffer: the operators leave it unused.
__device__ __forceinline__ bool plan_is_for(const int* head, int B, int N) {
  return ldg(head + PLAN_REQUESTS) == B && ldg(head + PLAN_ROWS) == N;
}

inline int plan_max_units(int B) { return B + kSplitRuns; }
inline size_t plan_part_rows(int n_rows) { return (size_t)n_rows + (n_rows > kSplitRows ? n_rows : kSplitRows); }

struct PlanLayout {
  size_t head, status, req, units, slot, position, row_req, mask, rope, total;
  PlanLayout(int B, int N, int Dh) {
    size_t o = 0;
    auto take = [&](size_t bytes) {
      const size_t at = o;
      o = align_up(o + bytes, 256);
      return at;
    };
    head = take(PLAN_WORDS * 4);
    status = take((size_t)B * 4);
    req = take((size_t)B * sizeof(BatchRequest));
    units = take((size_t)plan_max_units(B) * sizeof(BatchUnit));
    slot = take((size_t)N * 4);
    position = take((size_t)N * 4);
    row_req = take((size_t)N * 4);  // the row's request, -1: none
    mask = take((size_t)N * 16);
    rope = take((size_t)N * Dh * 4);
    total = o;
  }
};

struct PlanArgs {
  const int* row_start;  // [B + 1]
  const int* held;       // [B]
  const int* parent;     // [N] or null (chains)
  int* table;            // [B][max_pages]
  const int* free_pages; // [n_free]
  int B, N, max_pages, n_free, n_pages, prefix_len, Dh;
  double log2_theta;
  int* head;
  int* status;
  BatchRequest* req;
  BatchUnit* units;
  int* slot;
  int* position;
  int* row_req;
  uint32_t* mask;
  float* rope;
};
hipError_t launch_batch_plan(const PlanArgs& a, hipStream_t st);

struct StoreArgs {
  const bf16* q;
  const bf16* k;
  const bf16* v;
  long long q_stride, k_stride, v_stride;  // elements between rows
  bf16* q_out;                             // [N][H][Dh]
  bf16* k_pages;                           // the layer's pages [n_pages][Hkv][64][Dh]
  bf16* v_pages;                           // [n_pages][Hkv][Dh][64]
  const int* head;
  const int* slot;
  const float* rope;
  int B, N, H, Hkv, Dh, n_pages;
  int heads_per;  // heads that a workgroup turns (the launch sets it)
  int dim_parts;  // workgroups that share a head's values (the launch sets it)
  // llmcad_batch_norm_store alone
  const bf16* q_gain;  // null: ones
  const bf16* k_gain;
  long long q_gain_stride, k_gain_stride;  // elements between heads (0: one gain for all)
  float eps;
};
hipError_t launch_batch_store(const StoreArgs& a, hipStream_t st);
hipError_t launch_batch_norm_store(const StoreArgs& a, hipStream_t st);

struct CommitArgs {
  bf16* k_pages;  // [L][n_pages][Hkv][64][Dh]
  bf16* v_pages;
  const int* path;        // [N]
  const int* accept_len;  // [B]
  const int* head;
  const BatchRequest* req;
  const int* slot;
  int B, N, L, Hkv, Dh, n_pages;
  int heads_per;  // K/V heads per workgroup
};
hipError_t launch_batch_commit(const CommitArgs& a, hipStream_t st);

struct AttnArgs {
  const bf16* q;
  long long q_stride;
  const bf16* kc;  // the layer's prefix: K [Hkv][cap][Dh], V^T [Hkv][Dh][cap]
  const bf16* vc;
  int cap, P;
  const bf16* kp;  // the layer's pages
  const bf16* vp;
  int n_pages;
  const int* table;
  int max_pages;
  const int* head;
  const BatchRequest* req;
  const BatchUnit* units;
  const int* row_req;
  const uint32_t* mask;
  bf16* out;       // [N][H][Dh]
  float* part_o;   // partial results, unnormalised: [(KP N + partial rows)][H][Dh]
  float* part_ml;  // their running maximum (log2 domain) and sum [..][H][2]
  int B, N, H, Hkv, Dh;
  float scale_log2;
  int KP;     // key splits of the prefix
  int merge;  // runs of a request's pages per workgroup
};
hipError_t launch_batch_attention(const AttnArgs& a, hipStream_t st);
// Key splits of the prefix (the workspace holds max_prefix_splits(N) at most).
int prefix_splits(int N, int H, int Hkv, int P);
inline int max_prefix_splits(int N) { return N >= 1024 ? 2 : cdiv(2048, N) < 64 ? cdiv(2048, N) : 64; }

struct ScoresArgs {
  const void* logits;
  int bf16_in;
  long long stride;  // elements between rows
  int n, V, k, m;
  const int* tokens;  // [m]
  const int* row_of;  // [m] or null (m == n, token r under row r)
  float* logprob;     // [m]
  float* entropy;     // [n]
  float* lse;         // [n]
  int* top_token;     // [n][k]
  float* top_logprob; // [n][k]
  int parts, span;    // a row in workgroups of so many values
  float* part_sums;   // [n][parts][4]
  uint64_t* part_best; // [n][parts][k]
  float* row_scores;   // [n][4] where a second launch takes the tokens, else null
};
size_t score_work_bytes(int n, int V, int k);
hipError_t launch_token_scores(ScoresArgs a, void* workspace, hipStream_t st);

// Tokens of the vocabulary that a workgroup of the logits' adjustment takes at a time, and its threads.
constexpr int kAdjustChunk = 4096, kAdjustThreads = 512;

struct AdjustArgs {
  const void* logits;
  int bf16_in;
  long long stride, out_stride;  // elements between rows
  void* out;                     // null: not wanted
  int* greedy;                   // [N], null: not wanted
  llmcad_adjustments by;
  const int* head;
  const BatchRequest* req;
  const int* row_req;
  const uint32_t* mask;
  int B, N, V;
  int chunks;                // pieces of a row
  int chunks_per, rows_per;  // a workgroup's pieces (0: one, of several rows) and rows (the launch sets them)
  int segments;              // workgroups that share a row
  uint64_t* part;            // [N][segments][waves]: the best of each one's pieces
};
hipError_t launch_batch_adjust(const AdjustArgs& a, hipStream_t st);

struct AcceptArgs {
  const int* head;
  const BatchRequest* req;
  const uint32_t* mask;
  const int* tokens;  // [N]
  const int* greedy;  // [N]
  int* path;          // [N]
  int* accept_len;    // [B]
  int* next_token;    // [B]
  int* history;       // [B][history_stride] or null
  long long history_stride;
  int B, N;
};
hipError_t launch_batch_accept(const AcceptArgs& a, hipStream_t st);

// A page, or its first rows, that fork or compact copies to another.
struct PageCopy {
  int src, dst, rows;
};
struct PagesArgs {
  bf16* k_pages;  // [L][n_pages][Hkv][64][Dh]
  bf16* v_pages;
  int L, Hkv, Dh, n_pages;
  int B, max_pages;
  const int* table;   // [B][max_pages]
  const int* held;    // [B]
  const int* source;  // [B], fork alone
  int* table_out;     // [B][max_pages]
  int* held_out;      // [B], fork alone
  int* free_pages;    // [n_pages], fork alone
  int* n_free;        // fork alone
  int* status;        // fork alone
  int* n_used;        // compact alone
  int* n_copies;      // in the workspace, before the copies
  PageCopy* copies;
};
inline size_t pages_work_bytes(int B, int n_pages) {
  return 256 + align_up(sizeof(PageCopy) * (size_t)(B > n_pages / 2 ? B : n_pages / 2), 256);
}
hipError_t launch_batch_fork(const PagesArgs& a, hipStream_t st);
hipError_t launch_batch_compact(const PagesArgs& a, hipStream_t st);

}  // namespace llmcad
