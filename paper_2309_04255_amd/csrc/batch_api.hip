// Host side of the operators for several requests behind one shared prefix,
// and of the token scores: argument checks and launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include "batch.h"
#include "llmcad.h"

using namespace llmcad;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
template <typename... P>
bool aligned4(P... p) {
  return ((... | (uintptr_t)p) & 3) == 0;
}

// (Limits that keep every product below in 64 bits and every slot in 32.)
constexpr int kMaxRows = kMaxRequests * LLMCAD_MAX_NODES * 2;
constexpr int kMaxPages = (1 << 25) - 1;

int check_batch(const llmcad_config* cfg, int32_t n_requests, int32_t n_rows) {
  const int rc = llmcad_check_config(cfg);
  if (rc != LLMCAD_OK) return rc;
  if (n_requests < 1 || n_requests > kMaxRequests || n_rows < 1 || n_rows > kMaxRows) return LLMCAD_EARG;
  return LLMCAD_OK;
}

int check_kv_heads(const llmcad_config* cfg, int32_t n_kv_heads) {
  if (n_kv_heads < 1) return LLMCAD_EARG;
  return cfg->n_heads % n_kv_heads == 0 ? LLMCAD_OK : LLMCAD_ESHAPE;
}

int launched(hipError_t e) {
  if (e == hipSuccess) return LLMCAD_OK;
  keep_hip_error(e);
  return LLMCAD_EHIP;
}

size_t attn_part_rows(int n_rows) { return plan_part_rows(n_rows) + (size_t)max_prefix_splits(n_rows) * n_rows; }
size_t attn_ml_bytes(const llmcad_config* cfg, int n_rows) {
  return align_up(attn_part_rows(n_rows) * cfg->n_heads * 8, 256);
}

// The checks and arguments of a store.
int store_args(const llmcad_config* cfg, int32_t n_kv_heads, int32_t layer, const void* q, int64_t q_stride, const void* k,
               int64_t k_stride, const void* v, int64_t v_stride, void* q_out, void* k_pages, void* v_pages,
               int32_t n_pages, const void* plan, size_t plan_bytes, int32_t n_requests, int32_t n_rows, StoreArgs& a) {
  int rc = check_batch(cfg, n_requests, n_rows);
  if (rc != LLMCAD_OK) return rc;
  rc = check_kv_heads(cfg, n_kv_heads);
  if (rc != LLMCAD_OK) return rc;
  if (!q || !k || !v || !q_out || !k_pages || !v_pages || !plan || layer < 0 || layer >= cfg->n_layers || n_pages < 1 ||
      n_pages > kMaxPages)
    return LLMCAD_EARG;
  const int64_t H = cfg->n_heads, Hkv = n_kv_heads, Dh = cfg->head_dim;
  if (q_stride < H * Dh || k_stride < Hkv * Dh || v_stride < Hkv * Dh) return LLMCAD_ESHAPE;
  if (q_stride % 8 || k_stride % 8 || v_stride % 8 || !aligned16(q) || !aligned16(k) || !aligned16(v) ||
      !aligned16(q_out) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(plan))
    return LLMCAD_EARG;
  const PlanLayout P(n_requests, n_rows, cfg->head_dim);
  if (plan_bytes < P.total) return LLMCAD_EWORKSPACE;
  const size_t layer_at = (size_t)layer * n_pages * Hkv * kPage * Dh;
  a.q = (const bf16*)q;
  a.k = (const bf16*)k;
  a.v = (const bf16*)v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out = (bf16*)q_out;
  a.k_pages = (bf16*)k_pages + layer_at;
  a.v_pages = (bf16*)v_pages + layer_at;
  a.head = (const int*)((const char*)plan + P.head);
  a.slot = (const int*)((const char*)plan + P.slot);
  a.rope = (const float*)((const char*)plan + P.rope);
  a.B = n_requests;
  a.N = n_rows;
  a.H = cfg->n_heads;
  a.Hkv = n_kv_heads;
  a.Dh = cfg->head_dim;
  a.n_pages = n_pages;
  a.heads_per = a.dim_parts = 0;
  a.q_gain = a.k_gain = nullptr;
  a.q_gain_stride = a.k_gain_stride = 0;
  a.eps = 0.0f;
  return LLMCAD_OK;
}

// Whether n bytes from a on and m bytes from b on have one in common.
bool overlap(const void* a, size_t n, const void* b, size_t m) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + m && y < x + n;
}

// The checks and arguments that fork and compact have in common.
int pages_args(const llmcad_config* cfg, int32_t n_kv_heads, void* k_pages, void* v_pages, int32_t n_pages,
               int32_t n_requests, const int32_t* block_table, int32_t max_pages, const int32_t* held, int32_t* table_out,
               void* workspace, size_t workspace_bytes, PagesArgs& a) {
  int rc = check_batch(cfg, n_requests, 1);
  if (rc != LLMCAD_OK) return rc;
  rc = check_kv_heads(cfg, n_kv_heads);
  if (rc != LLMCAD_OK) return rc;
  if (!k_pages || !v_pages || !block_table || !held || !table_out || !workspace || n_pages < 1 || n_pages > LLMCAD_MAX_POOL ||
      max_pages < 1 || max_pages > LLMCAD_MAX_POOL || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(workspace) ||
      !aligned4(block_table, held, table_out))
    return LLMCAD_EARG;
  const size_t table = (size_t)n_requests * max_pages * 4, lengths = (size_t)n_requests * 4;
  if (overlap(table_out, table, block_table, table) || overlap(table_out, table, held, lengths)) return LLMCAD_EARG;
  if (workspace_bytes < pages_work_bytes(n_requests, n_pages)) return LLMCAD_EWORKSPACE;
  a = PagesArgs{};
  a.k_pages = (bf16*)k_pages;
  a.v_pages = (bf16*)v_pages;
  a.L = cfg->n_layers;
  a.Hkv = n_kv_heads;
  a.Dh = cfg->head_dim;
  a.n_pages = n_pages;
  a.B = n_requests;
  a.max_pages = max_pages;
  a.table = block_table;
  a.held = held;
  a.table_out = table_out;
  a.n_copies = (int*)workspace;
  a.copies = (PageCopy*)((char*)workspace + 256);
  return LLMCAD_OK;
}

}  // namespace

extern "C" {

size_t llmcad_batch_plan_bytes(const llmcad_config* cfg, int32_t n_requests, int32_t n_rows) {
  if (check_batch(cfg, n_requests, n_rows) != LLMCAD_OK) return 0;
  return PlanLayout(n_requests, n_rows, cfg->head_dim).total;
}

int llmcad_batch_plan_region(const llmcad_config* cfg, int32_t n_requests, int32_t n_rows, int32_t which, size_t* offset,
                             size_t* bytes) {
  const int rc = check_batch(cfg, n_requests, n_rows);
  if (rc != LLMCAD_OK) return rc;
  if (!offset || !bytes) return LLMCAD_EARG;
  const PlanLayout P(n_requests, n_rows, cfg->head_dim);
  const size_t N = (size_t)n_rows;
  switch (which) {
    case 0: *offset = P.slot; *bytes = N * 4; break;
    case 1: *offset = P.position; *bytes = N * 4; break;
    case 2: *offset = P.mask; *bytes = N * 16; break;
    case 3: *offset = P.rope; *bytes = N * cfg->head_dim * 4; break;
    case 4: *offset = P.status; *bytes = (size_t)n_requests * 4; break;
    case 5: *offset = P.head + PLAN_TAKEN * 4; *bytes = 4; break;
    default: return LLMCAD_EARG;
  }
  return LLMCAD_OK;
}

int llmcad_batch_plan(const llmcad_config* cfg, int32_t n_requests, int32_t n_rows, const int32_t* row_start,
                      const int32_t* held, const int32_t* parent, int32_t prefix_len, int32_t* block_table,
                      int32_t max_pages, const int32_t* free_pages, int32_t n_free, int32_t n_pages, void* plan,
                      size_t plan_bytes, void* stream) {
  const int rc = check_batch(cfg, n_requests, n_rows);
  if (rc != LLMCAD_OK) return rc;
  if (!row_start || !held || !block_table || !plan || !aligned16(plan) || max_pages < 1 || max_pages > kMaxPages ||
      n_pages < 1 || n_pages > kMaxPages || n_free < 0 || (n_free > 0 && !free_pages) ||
      !aligned4(row_start, held, parent, block_table, free_pages))
    return LLMCAD_EARG;
  if (prefix_len < 0 || prefix_len > (1 << 30)) return LLMCAD_ECAPACITY;
  const PlanLayout P(n_requests, n_rows, cfg->head_dim);
  if (plan_bytes < P.total) return LLMCAD_EWORKSPACE;
  char* at = (char*)plan;
  PlanArgs a;
  a.row_start = row_start;
  a.held = held;
  a.parent = parent;
  a.table = block_table;
  a.free_pages = free_pages;
  a.B = n_requests;
  a.N = n_rows;
  a.max_pages = max_pages;
  a.n_free = n_free;
  a.n_pages = n_pages;
  a.prefix_len = prefix_len;
  a.Dh = cfg->head_dim;
  a.log2_theta = log2((double)cfg->rope_theta);
  a.head = (int*)(at + P.head);
  a.status = (int*)(at + P.status);
  a.req = (BatchRequest*)(at + P.req);
  a.units = (BatchUnit*)(at + P.units);
  a.slot = (int*)(at + P.slot);
  a.position = (int*)(at + P.position);
  a.row_req = (int*)(at + P.row_req);
  a.mask = (uint32_t*)(at + P.mask);
  a.rope = (float*)(at + P.rope);
  return launched(launch_batch_plan(a, (hipStream_t)stream));
}

int llmcad_batch_store(const llmcad_config* cfg, int32_t n_kv_heads, int32_t layer, const void* q, int64_t q_stride,
                       const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out, void* k_pages,
                       void* v_pages, int32_t n_pages, const void* plan, size_t plan_bytes, int32_t n_requests,
                       int32_t n_rows, void* stream) {
  StoreArgs a;
  const int rc = store_args(cfg, n_kv_heads, layer, q, q_stride, k, k_stride, v, v_stride, q_out, k_pages, v_pages, n_pages,
                            plan, plan_bytes, n_requests, n_rows, a);
  return rc != LLMCAD_OK ? rc : launched(launch_batch_store(a, (hipStream_t)stream));
}

int llmcad_batch_norm_store(const llmcad_config* cfg, int32_t n_kv_heads, int32_t layer, const void* q, int64_t q_stride,
                            const void* k, int64_t k_stride, const void* v, int64_t v_stride, const void* q_gain,
                            int64_t q_gain_stride, const void* k_gain, int64_t k_gain_stride, void* q_out, void* k_pages,
                            void* v_pages, int32_t n_pages, const void* plan, size_t plan_bytes, int32_t n_requests,
                            int32_t n_rows, void* stream) {
  StoreArgs a;
  const int rc = store_args(cfg, n_kv_heads, layer, q, q_stride, k, k_stride, v, v_stride, q_out, k_pages, v_pages, n_pages,
                            plan, plan_bytes, n_requests, n_rows, a);
  if (rc != LLMCAD_OK) return rc;
  const int64_t Dh = cfg->head_dim;
  if (!aligned16(q_gain) || !aligned16(k_gain) || q_gain_stride % 8 || k_gain_stride % 8) return LLMCAD_EARG;
  if ((q_gain_stride != 0 && q_gain_stride < Dh) || (k_gain_stride != 0 && k_gain_stride < Dh)) return LLMCAD_ESHAPE;
  a.q_gain = (const bf16*)q_gain;
  a.k_gain = (const bf16*)k_gain;
  a.q_gain_stride = q_gain_stride;
  a.k_gain_stride = k_gain_stride;
  a.eps = cfg->rms_eps;
  return launched(launch_batch_norm_store(a, (hipStream_t)stream));
}

size_t llmcad_batch_workspace_bytes(const llmcad_config* cfg, int32_t n_kv_heads, int32_t n_requests, int32_t n_rows) {
  if (check_batch(cfg, n_requests, n_rows) != LLMCAD_OK || check_kv_heads(cfg, n_kv_heads) != LLMCAD_OK) return 0;
  return attn_ml_bytes(cfg, n_rows) + attn_part_rows(n_rows) * cfg->n_heads * cfg->head_dim * 4;
}

int llmcad_batch_attention(const llmcad_config* cfg, int32_t n_kv_heads, int32_t layer, const void* q, int64_t q_stride,
                           const void* k_cache, const void* v_cache, int32_t capacity, int32_t prefix_len,
                           const void* k_pages, const void* v_pages, int32_t n_pages, const int32_t* block_table,
                           int32_t max_pages, const void* plan, size_t plan_bytes, int32_t n_requests, int32_t n_rows,
                           void* out, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_batch(cfg, n_requests, n_rows);
  if (rc != LLMCAD_OK) return rc;
  rc = check_kv_heads(cfg, n_kv_heads);
  if (rc != LLMCAD_OK) return rc;
  if (!q || !k_pages || !v_pages || !block_table || !plan || !out || !workspace || layer < 0 || layer >= cfg->n_layers ||
      n_pages < 1 || n_pages > kMaxPages || max_pages < 1 || max_pages > kMaxPages)
    return LLMCAD_EARG;
  if (prefix_len < 0) return LLMCAD_ECAPACITY;
  if (prefix_len > 0) {
    if (!k_cache || !v_cache || !aligned16(k_cache) || !aligned16(v_cache)) return LLMCAD_EARG;
    // (the offset of a value within a head's V^T is 32 bits)
    if (capacity < 64 || capacity % 64 != 0 || capacity > (1 << 24) || prefix_len > capacity) return LLMCAD_ECAPACITY;
  }
  const int64_t H = cfg->n_heads, Dh = cfg->head_dim;
  if (q_stride < H * Dh) return LLMCAD_ESHAPE;
  if (q_stride % 8 || !aligned16(q) || !aligned16(out) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(plan) ||
      !aligned16(workspace) || !aligned4(block_table))
    return LLMCAD_EARG;
  const PlanLayout P(n_requests, n_rows, cfg->head_dim);
  if (plan_bytes < P.total || workspace_bytes < llmcad_batch_workspace_bytes(cfg, n_kv_heads, n_requests, n_rows))
    return LLMCAD_EWORKSPACE;
  const char* at = (const char*)plan;
  const size_t page_at = (size_t)layer * n_pages * n_kv_heads * kPage * Dh;
  const size_t cache_at = (size_t)layer * n_kv_heads * capacity * Dh;
  AttnArgs a;
  a.q = (const bf16*)q;
  a.q_stride = q_stride;
  a.kc = prefix_len > 0 ? (const bf16*)k_cache + cache_at : nullptr;
  a.vc = prefix_len > 0 ? (const bf16*)v_cache + cache_at : nullptr;
  a.cap = capacity;
  a.P = prefix_len;
  a.kp = (const bf16*)k_pages + page_at;
  a.vp = (const bf16*)v_pages + page_at;
  a.n_pages = n_pages;
  a.table = block_table;
  a.max_pages = max_pages;
  a.head = (const int*)(at + P.head);
  a.req = (const BatchRequest*)(at + P.req);
  a.units = (const BatchUnit*)(at + P.units);
  a.row_req = (const int*)(at + P.row_req);
  a.mask = (const uint32_t*)(at + P.mask);
  a.out = (bf16*)out;
  a.part_ml = (float*)workspace;
  a.part_o = (float*)((char*)workspace + attn_ml_bytes(cfg, n_rows));
  a.B = n_requests;
  a.N = n_rows;
  a.H = cfg->n_heads;
  a.Hkv = n_kv_heads;
  a.Dh = cfg->head_dim;
  a.scale_log2 = (float)(1.4426950408889634 / sqrt((double)cfg->head_dim));
  a.KP = prefix_splits(n_rows, cfg->n_heads, n_kv_heads, prefix_len);
  return launched(launch_batch_attention(a, (hipStream_t)stream));
}

int llmcad_batch_commit(const llmcad_config* cfg, int32_t n_kv_heads, void* k_pages, void* v_pages, int32_t n_pages,
                        const void* plan, size_t plan_bytes, int32_t n_requests, int32_t n_rows, const int32_t* path,
                        const int32_t* accept_len, void* stream) {
  int rc = check_batch(cfg, n_requests, n_rows);
  if (rc != LLMCAD_OK) return rc;
  rc = check_kv_heads(cfg, n_kv_heads);
  if (rc != LLMCAD_OK) return rc;
  if (!k_pages || !v_pages || !plan || !path || !accept_len || n_pages < 1 || n_pages > kMaxPages || !aligned16(k_pages) ||
      !aligned16(v_pages) || !aligned16(plan) || !aligned4(path, accept_len))
    return LLMCAD_EARG;
  const PlanLayout P(n_requests, n_rows, cfg->head_dim);
  if (plan_bytes < P.total) return LLMCAD_EWORKSPACE;
  CommitArgs a;
  a.k_pages = (bf16*)k_pages;
  a.v_pages = (bf16*)v_pages;
  a.path = path;
  a.accept_len = accept_len;
  a.head = (const int*)((const char*)plan + P.head);
  a.req = (const BatchRequest*)((const char*)plan + P.req);
  a.slot = (const int*)((const char*)plan + P.slot);
  a.B = n_requests;
  a.N = n_rows;
  a.L = cfg->n_layers;
  a.Hkv = n_kv_heads;
  a.Dh = cfg->head_dim;
  a.n_pages = n_pages;
  return launched(launch_batch_commit(a, (hipStream_t)stream));
}

size_t llmcad_batch_adjust_workspace_bytes(const llmcad_config* cfg, int32_t n_rows) {
  if (check_batch(cfg, 1, n_rows) != LLMCAD_OK) return 0;
  return align_up((size_t)n_rows * cdiv(cfg->vocab, kAdjustChunk) * (kAdjustThreads / kWave) * 8, 256);
}

int llmcad_batch_adjust(const llmcad_config* cfg, const void* plan, size_t plan_bytes, int32_t n_requests, int32_t n_rows,
                        const void* logits, int32_t bits, int64_t row_stride, const llmcad_adjustments* by, void* out,
                        int64_t out_stride, int32_t* greedy, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_batch(cfg, n_requests, n_rows);
  if (rc != LLMCAD_OK) return rc;
  if (!plan || !aligned16(plan) || !logits || (bits != 16 && bits != 32) || !by || (!out && !greedy) || !workspace ||
      !aligned16(workspace))
    return LLMCAD_EARG;
  const uintptr_t element = bits / 8;
  if ((uintptr_t)logits % element || (uintptr_t)out % element ||
      !aligned4(greedy, by->tokens, by->history, by->prompt_len, by->seen, by->penalties, by->bias_start, by->bias_token,
                by->bias_value, by->allow, by->mask_of))
    return LLMCAD_EARG;
  if ((by->penalties && !by->tokens) || (by->history && by->history_stride < 0) ||
      (by->bias_start && (by->n_bias < 0 || (by->n_bias > 0 && (!by->bias_token || !by->bias_value)))) ||
      (by->allow && by->n_masks < 1) ||
      (!by->allow != !by->mask_of))
    return LLMCAD_EARG;
  if (row_stride < cfg->vocab || (out && out_stride < cfg->vocab)) return LLMCAD_ESHAPE;
  // (in place every element is read by the thread that writes it, if the rows are the same ones)
  if (out && !(out == logits && (out_stride == row_stride || n_rows == 1))) {
    const size_t V = (size_t)cfg->vocab, rows = (size_t)n_rows - 1;
    if (overlap(out, (rows * out_stride + V) * element, logits, (rows * row_stride + V) * element)) return LLMCAD_EARG;
  }
  const PlanLayout P(n_requests, n_rows, cfg->head_dim);
  if (plan_bytes < P.total || workspace_bytes < llmcad_batch_adjust_workspace_bytes(cfg, n_rows)) return LLMCAD_EWORKSPACE;
  const char* at = (const char*)plan;
  AdjustArgs a;
  a.logits = logits;
  a.bf16_in = bits == 16;
  a.stride = row_stride;
  a.out_stride = out_stride;
  a.out = out;
  a.greedy = greedy;
  a.by = *by;
  a.head = (const int*)(at + P.head);
  a.req = (const BatchRequest*)(at + P.req);
  a.row_req = (const int*)(at + P.row_req);
  a.mask = (const uint32_t*)(at + P.mask);
  a.B = n_requests;
  a.N = n_rows;
  a.V = cfg->vocab;
  a.chunks = a.chunks_per = a.rows_per = a.segments = 0;
  a.part = (uint64_t*)workspace;
  return launched(launch_batch_adjust(a, (hipStream_t)stream));
}

int llmcad_batch_accept(const llmcad_config* cfg, const void* plan, size_t plan_bytes, int32_t n_requests, int32_t n_rows,
                        const int32_t* tokens, const int32_t* greedy, int32_t* path, int32_t* accept_len,
                        int32_t* next_token, int32_t* history, int64_t history_stride, void* stream) {
  const int rc = check_batch(cfg, n_requests, n_rows);
  if (rc != LLMCAD_OK) return rc;
  if (!plan || !aligned16(plan) || !tokens || !greedy || !path || !accept_len || !next_token ||
      (history && history_stride < 0) || !aligned4(tokens, greedy, path, accept_len, next_token, history))
    return LLMCAD_EARG;
  const PlanLayout P(n_requests, n_rows, cfg->head_dim);
  if (plan_bytes < P.total) return LLMCAD_EWORKSPACE;
  // (a thread writes an entry of the path while another still reads its token)
  const size_t rows = (size_t)n_rows * 4, requests = (size_t)n_requests * 4;
  const struct {
    const void* at;
    size_t bytes;
  } outs[] = {{path, rows}, {accept_len, requests}, {next_token, requests}, {history, history ? requests * (size_t)history_stride : 0}};
  for (const auto& o : outs)
    if (o.bytes && (overlap(o.at, o.bytes, tokens, rows) || overlap(o.at, o.bytes, greedy, rows))) return LLMCAD_EARG;
  const char* at = (const char*)plan;
  AcceptArgs a;
  a.head = (const int*)(at + P.head);
  a.req = (const BatchRequest*)(at + P.req);
  a.mask = (const uint32_t*)(at + P.mask);
  a.tokens = tokens;
  a.greedy = greedy;
  a.path = path;
  a.accept_len = accept_len;
  a.next_token = next_token;
  a.history = history;
  a.history_stride = history_stride;
  a.B = n_requests;
  a.N = n_rows;
  return launched(launch_batch_accept(a, (hipStream_t)stream));
}

size_t llmcad_batch_pages_workspace_bytes(int32_t n_requests, int32_t n_pages) {
  if (n_requests < 1 || n_requests > kMaxRequests || n_pages < 1 || n_pages > LLMCAD_MAX_POOL) return 0;
  return pages_work_bytes(n_requests, n_pages);
}

int llmcad_batch_fork(const llmcad_config* cfg, int32_t n_kv_heads, void* k_pages, void* v_pages, int32_t n_pages,
                      int32_t n_requests, const int32_t* block_table, int32_t max_pages, const int32_t* held,
                      const int32_t* source, int32_t* table_out, int32_t* held_out, int32_t* free_pages, int32_t* n_free,
                      int32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
  PagesArgs a;
  const int rc = pages_args(cfg, n_kv_heads, k_pages, v_pages, n_pages, n_requests, block_table, max_pages, held, table_out,
                            workspace, workspace_bytes, a);
  if (rc != LLMCAD_OK) return rc;
  if (!source || !held_out || !free_pages || !n_free || !status || !aligned4(source, held_out, free_pages, n_free, status))
    return LLMCAD_EARG;
  const size_t table = (size_t)n_requests * max_pages * 4, lengths = (size_t)n_requests * 4;
  const struct {
    const void* at;
    size_t bytes;
  } outs[] = {{table_out, table}, {held_out, lengths}, {free_pages, (size_t)n_pages * 4}, {n_free, 4}, {status, 4}};
  for (const auto& o : outs)
    if (overlap(o.at, o.bytes, block_table, table) || overlap(o.at, o.bytes, held, lengths) ||
        overlap(o.at, o.bytes, source, lengths))
      return LLMCAD_EARG;
  a.source = source;
  a.held_out = held_out;
  a.free_pages = free_pages;
  a.n_free = n_free;
  a.status = status;
  return launched(launch_batch_fork(a, (hipStream_t)stream));
}

int llmcad_batch_compact(const llmcad_config* cfg, int32_t n_kv_heads, void* k_pages, void* v_pages, int32_t n_pages,
                         int32_t n_requests, const int32_t* block_table, int32_t max_pages, const int32_t* held,
                         int32_t* table_out, int32_t* n_used, void* workspace, size_t workspace_bytes, void* stream) {
  PagesArgs a;
  const int rc = pages_args(cfg, n_kv_heads, k_pages, v_pages, n_pages, n_requests, block_table, max_pages, held, table_out,
                            workspace, workspace_bytes, a);
  if (rc != LLMCAD_OK) return rc;
  const size_t table = (size_t)n_requests * max_pages * 4;
  if (!n_used || !aligned4(n_used) || overlap(n_used, 4, block_table, table) || overlap(n_used, 4, held, (size_t)n_requests * 4))
    return LLMCAD_EARG;
  a.n_used = n_used;
  return launched(launch_batch_compact(a, (hipStream_t)stream));
}

size_t llmcad_token_scores_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t k) {
  if (n_rows < 1 || n_rows >= (1 << 24) || vocab < 1 || vocab > (1 << 24) || k < 0 || k > LLMCAD_TOP_MAX) return 0;
  return std::max((size_t)256, score_work_bytes(n_rows, vocab, k));
}

int llmcad_token_scores(const void* logits, int32_t bits, int64_t row_stride, int32_t n_rows, int32_t vocab,
                        const int32_t* tokens, const int32_t* row_of, int32_t n_tokens, float* logprob, float* entropy,
                        float* lse, int32_t k, int32_t* top_token, float* top_logprob, void* workspace,
                        size_t workspace_bytes, void* stream) {
  if (!logits || !entropy || !lse || !workspace || (bits != 16 && bits != 32) || n_rows < 1 || vocab < 1 || n_tokens < 0 ||
      (n_tokens > 0 && (!tokens || !logprob)) || (n_tokens > 0 && !row_of && n_tokens != n_rows) || k < 0 ||
      k > LLMCAD_TOP_MAX || (k > 0 && (!top_token || !top_logprob)))
    return LLMCAD_EARG;
  // (more rows than a launch takes workgroups of 256 threads; a workgroup counts the tokens in 32 bits, past the last)
  if (n_rows >= (1 << 24) || n_tokens > (1 << 30)) return LLMCAD_EARG;
  if (row_stride < vocab || vocab > (1 << 24)) return LLMCAD_ESHAPE;
  if (((uintptr_t)logits & (bits / 8 - 1)) != 0 || !aligned16(workspace) ||
      !aligned4(tokens, row_of, logprob, entropy, lse, top_token, top_logprob))
    return LLMCAD_EARG;
  if (workspace_bytes < llmcad_token_scores_workspace_bytes(n_rows, vocab, k)) return LLMCAD_EWORKSPACE;
  ScoresArgs a;
  a.logits = logits;
  a.bf16_in = bits == 16;
  a.stride = row_stride;
  a.n = n_rows;
  a.V = vocab;
  a.k = k;
  a.m = n_tokens;
  a.tokens = tokens;
  a.row_of = row_of;
  a.logprob = logprob;
  a.entropy = entropy;
  a.lse = lse;
  a.top_token = top_token;
  a.top_logprob = top_logprob;
  return launched(launch_token_scores(a, workspace, (hipStream_t)stream));
}

}  // extern "C"
