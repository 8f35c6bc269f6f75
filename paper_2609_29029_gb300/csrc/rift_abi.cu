// The C ABI of include/rift.h: argument validation, workspace carving and launches on the
// caller's stream.  Nothing here allocates device memory.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <mutex>
#include <vector>

#include "kv_pages.cuh"
#include "rift_internal.h"

using namespace rift;

namespace {

constexpr size_t WS_ALIGN = 256;

bool ws_ok(const void* ws, size_t have, size_t need) {
  if (need == 0) return true;
  return ws != nullptr && have >= need && (reinterpret_cast<uintptr_t>(ws) % WS_ALIGN) == 0;
}

bool dims_ok(int N, int n_v, int d) {
  return N >= 1 && N <= RIFT_MAX_TILES && n_v >= 1 && n_v <= RIFT_MAX_NV && d >= 64 && d <= 8192 &&
         d % 64 == 0;
}

struct ProfRec {
  int cls, n;
  cudaEvent_t a, b;
};
std::mutex g_prof_mu;
bool g_prof_on = false;
std::vector<cudaEvent_t> g_pool;
std::vector<ProfRec> g_recs;
cudaEvent_t g_open[RIFT_PROF_CLASSES] = {};
std::atomic<long long> g_launches{0};
// Set by the first call of the paged cache: rift_sync_status reads those flags (two more round trips each)
// only in processes that use it.
std::atomic<bool> g_paged_used{false};

cudaEvent_t pool_get() {
  if (!g_pool.empty()) {
    cudaEvent_t e = g_pool.back();
    g_pool.pop_back();
    return e;
  }
  cudaEvent_t e = nullptr;
  if (cudaEventCreate(&e) != cudaSuccess) return nullptr;
  return e;
}

}  // namespace

namespace rift {

unsigned long long current_context_id() {
  static PFN_cuCtxGetCurrent_v4000 get_current = nullptr;
  static PFN_cuCtxGetId_v12000 get_id = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuCtxGetCurrent", &p, 4000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      get_current = reinterpret_cast<PFN_cuCtxGetCurrent_v4000>(p);
    p = nullptr;
    if (cudaGetDriverEntryPointByVersion("cuCtxGetId", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      get_id = reinterpret_cast<PFN_cuCtxGetId_v12000>(p);
  });
  CUcontext ctx = nullptr;
  unsigned long long id = 0;
  if (!get_current || !get_id || get_current(&ctx) != CUDA_SUCCESS || !ctx || get_id(ctx, &id) != CUDA_SUCCESS)
    return 0;
  return id;
}

void prof_begin(int cls, cudaStream_t st) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  if (!g_prof_on) return;
  cudaEvent_t e = pool_get();
  if (e && cudaEventRecord(e, st) == cudaSuccess) g_open[cls] = e;
}

void prof_end(int cls, cudaStream_t st, int n) {
  g_launches += n;
  std::lock_guard<std::mutex> lk(g_prof_mu);
  if (!g_prof_on || !g_open[cls]) return;
  cudaEvent_t e = pool_get();
  if (e && cudaEventRecord(e, st) == cudaSuccess) g_recs.push_back({cls, n, g_open[cls], e});
  g_open[cls] = nullptr;
}

rift_status score_args_check(const void* X, rift_dtype xdt, int N, int n_v, int d, const float* t, const float* B,
                             int M, int knn_m, const float* token_scores, const float* tile_s_raw,
                             const float* tile_s) {
  if (!dims_ok(N, n_v, d) || !X || !t || !token_scores || !tile_s_raw || !tile_s) return RIFT_ERR_INVALID;
  if (xdt != RIFT_F32 && xdt != RIFT_BF16) return RIFT_ERR_INVALID;
  if (xdt == RIFT_F32 && d > 4096) return RIFT_ERR_UNSUPPORTED;
  if (M < 0 || M > 64 || (M > 0 && !B) || knn_m < 0 || knn_m > RIFT_MAX_KNN) return RIFT_ERR_INVALID;
  if (!aligned16(X)) return RIFT_ERR_INVALID;
  return RIFT_OK;
}

}  // namespace rift

extern "C" {

void rift_profile_enable(int on) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  g_prof_on = on != 0;
}

rift_status rift_profile_read(double* ms, long long* launches, int n_classes) {
  std::lock_guard<std::mutex> lk(g_prof_mu);
  rift_status st = RIFT_OK;
  for (int c = 0; c < n_classes; ++c) {
    if (ms) ms[c] = 0.0;
    if (launches) launches[c] = 0;
  }
  for (const ProfRec& r : g_recs) {
    float t = 0.f;
    if (cudaEventSynchronize(r.b) != cudaSuccess || cudaEventElapsedTime(&t, r.a, r.b) != cudaSuccess) st = RIFT_ERR_CUDA;
    if (r.cls < n_classes) {
      if (ms) ms[r.cls] += t;
      if (launches) launches[r.cls] += r.n;
    }
    g_pool.push_back(r.a);
    g_pool.push_back(r.b);
  }
  g_recs.clear();
  return st;
}

long long rift_launch_count(void) { return g_launches.load(); }

int rift_abi_version(void) { return 5; }

const char* rift_status_string(rift_status s) {
  switch (s) {
    case RIFT_OK: return "ok";
    case RIFT_ERR_INVALID: return "invalid argument";
    case RIFT_ERR_CAPACITY: return "output capacity exceeded";
    case RIFT_ERR_NONFINITE: return "non-finite score";
    case RIFT_ERR_CUDA: return "CUDA runtime error";
    case RIFT_ERR_TIMEOUT: return "device wait timed out";
    case RIFT_ERR_UNSUPPORTED: return "unsupported";
    case RIFT_ERR_BAD_ID: return "id out of range";
  }
  return "unknown status";
}

rift_status rift_sync_status(rift_stream_t stream) {
  if (cudaStreamSynchronize(static_cast<cudaStream_t>(stream)) != cudaSuccess) return RIFT_ERR_CUDA;
  unsigned int f = read_clear_err_score() | read_clear_err_select() | read_clear_err_pack() |
                   read_clear_err_prefill() | read_clear_err_gemm() | read_clear_err_attn() | read_clear_err_merge();
  if (g_paged_used.load()) f |= read_clear_err_kv() | read_clear_err_paged();
  if (cudaGetLastError() != cudaSuccess) return RIFT_ERR_CUDA;
  if (f & RIFT_EBIT_BADID) return RIFT_ERR_BAD_ID;
  if (f & RIFT_EBIT_NONFINITE) return RIFT_ERR_NONFINITE;
  if (f & RIFT_EBIT_CAPACITY) return RIFT_ERR_CAPACITY;
  if (f & RIFT_EBIT_TIMEOUT) return RIFT_ERR_TIMEOUT;
  return RIFT_OK;
}

rift_status rift_query_prep(const void* embed, int vocab, int d, const int* phrase_ids, int n_templates,
                            int n_phrase, const int* bg_ids, int M, float* t, float* B,
                            rift_stream_t stream) {
  if (!embed || !phrase_ids || !t || vocab < 1 || d < 64 || d > 8192 || d % 64 != 0 || n_templates < 1 ||
      n_phrase < 1 || M < 0 || M > 64 || (M > 0 && (!bg_ids || !B)))
    return RIFT_ERR_INVALID;
  prof_begin(RIFT_PROF_SCORE, static_cast<cudaStream_t>(stream));
  const int nk = launch_query_prep(embed, vocab, d, phrase_ids, n_templates, n_phrase, bg_ids, M, t, B,
                                   static_cast<cudaStream_t>(stream));
  prof_end(RIFT_PROF_SCORE, static_cast<cudaStream_t>(stream), nk);
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_score_workspace_bytes(int N, int n_v, int d, int M) {
  if (!dims_ok(N, n_v, d)) return 0;
  return score_layout(N, n_v, d, M).total;
}

rift_status rift_score_tiles(const void* X, rift_dtype xdt, int N, int n_v, int d, const float* t,
                             const float* B, int M, int knn_m, float* token_scores, float* tile_s_raw,
                             float* tile_s, int* nbr, void* ws, size_t ws_bytes, rift_stream_t stream) {
  const rift_status chk = score_args_check(X, xdt, N, n_v, d, t, B, M, knn_m, token_scores, tile_s_raw, tile_s);
  if (chk != RIFT_OK) return chk;
  const size_t need = rift_score_workspace_bytes(N, n_v, d, M);
  if (!ws_ok(ws, ws_bytes, need)) return RIFT_ERR_INVALID;
  const int m = std::min(knn_m, N - 1);
  prof_begin(RIFT_PROF_SCORE, static_cast<cudaStream_t>(stream));
  const int nk = launch_score(X, xdt, N, n_v, d, t, B, M, m, token_scores, tile_s_raw, tile_s, nbr,
                              static_cast<char*>(ws), static_cast<cudaStream_t>(stream));
  prof_end(RIFT_PROF_SCORE, static_cast<cudaStream_t>(stream), nk < 0 ? 0 : nk);
  if (nk < 0) return RIFT_ERR_CUDA;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_select_workspace_bytes(int N, int n_v) {
  (void)N;
  (void)n_v;
  return 0;
}

static rift_status select_args_check(const float* token_scores, const float* tile_s, int N, int n_v,
                                     const rift_policy* policy, const float* u, const int* kept, const int* n_kept,
                                     const int* budgets, const int* sel, const int* sel_off) {
  if (!token_scores || !tile_s || !policy || !u || !kept || !n_kept || !budgets || !sel || !sel_off)
    return RIFT_ERR_INVALID;
  if (N < 1 || N > RIFT_MAX_TILES || n_v < 1 || n_v > RIFT_MAX_NV) return RIFT_ERR_INVALID;
  const rift_policy& pol = *policy;
  if (!(pol.tau >= 0.f && pol.tau <= 1.f)) return RIFT_ERR_INVALID;
  if (pol.n_c < 1 || pol.n_c > RIFT_MAX_BUDGETS) return RIFT_ERR_INVALID;
  for (int c = 0; c < pol.n_c; ++c) {
    if (pol.C[c] < 1 || pol.C[c] > n_v) return RIFT_ERR_INVALID;
    if (c > 0 && pol.C[c] <= pol.C[c - 1]) return RIFT_ERR_INVALID;
    if (!std::isfinite(pol.alpha_pos[c]) || !std::isfinite(pol.alpha_neg[c]) || !std::isfinite(pol.energy[c]))
      return RIFT_ERR_INVALID;
  }
  if (!std::isfinite(pol.lambda)) return RIFT_ERR_INVALID;
  if (pol.ctx_num < 0 || pol.ctx_den < 1 || pol.ctx_num >= pol.ctx_den) return RIFT_ERR_INVALID;
  return RIFT_OK;
}

rift_status rift_select_budgeted_tokens(const float* token_scores, const float* tile_s, int N, int n_v,
                                        const float* p, const rift_policy* policy, float* u, int* kept,
                                        int* n_kept, int* budgets, int* sel, int* sel_off, void* ws,
                                        size_t ws_bytes, rift_stream_t stream) {
  (void)ws;
  (void)ws_bytes;
  const rift_status chk =
      select_args_check(token_scores, tile_s, N, n_v, policy, u, kept, n_kept, budgets, sel, sel_off);
  if (chk != RIFT_OK) return chk;
  prof_begin(RIFT_PROF_SELECT, static_cast<cudaStream_t>(stream));
  const int launches = launch_select(token_scores, tile_s, N, n_v, p, *policy, u, kept, n_kept, budgets, sel, sel_off,
                                     static_cast<cudaStream_t>(stream));
  prof_end(RIFT_PROF_SELECT, static_cast<cudaStream_t>(stream), launches);
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

// ---- one scene sharded over several ranks (a shard of its tiles per rank) ----

size_t rift_score_shard_workspace_bytes(int N_local, int n_v, int d) {
  if (!dims_ok(N_local, n_v, d)) return 0;
  return shard_layout(N_local, n_v, d).total;
}

rift_status rift_score_shard(const void* X, rift_dtype xdt, int N_local, int n_v, int d, const float* t,
                             const float* B, int M, float* token_scores, float* tile_s_raw, float* V, void* ws,
                             size_t ws_bytes, rift_stream_t stream) {
  if (!V) return RIFT_ERR_INVALID;
  const rift_status chk = score_args_check(X, xdt, N_local, n_v, d, t, B, M, 0, token_scores, tile_s_raw, V);
  if (chk != RIFT_OK) return chk;
  if (!ws_ok(ws, ws_bytes, rift_score_shard_workspace_bytes(N_local, n_v, d))) return RIFT_ERR_INVALID;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  prof_begin(RIFT_PROF_SCORE, st);
  const int nk = launch_score_tokens(X, xdt, N_local, n_v, d, t, B, M, token_scores, tile_s_raw, V,
                                     static_cast<char*>(ws), st);
  prof_end(RIFT_PROF_SCORE, st, nk);
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_smooth_workspace_bytes(int N, int n_rows, int d) {
  if (N < 1 || N > RIFT_MAX_TILES || n_rows < 1 || n_rows > N || d < 64 || d > 8192 || d % 64 != 0) return 0;
  return smooth_layout(N, n_rows, d).total;
}

rift_status rift_smooth_rows(const float* V, const float* tile_s_raw, int N, int d, int row0, int n_rows, int knn_m,
                             float* tile_s, int* nbr, void* ws, size_t ws_bytes, rift_stream_t stream) {
  if (!V || !tile_s_raw || !tile_s || N < 1 || N > RIFT_MAX_TILES || d < 64 || d > 8192 || d % 64 != 0)
    return RIFT_ERR_INVALID;
  if (row0 < 0 || n_rows < 1 || row0 + n_rows > N || knn_m < 0 || knn_m > RIFT_MAX_KNN) return RIFT_ERR_INVALID;
  if (!aligned16(V)) return RIFT_ERR_INVALID;
  if (!ws_ok(ws, ws_bytes, rift_smooth_workspace_bytes(N, n_rows, d))) return RIFT_ERR_INVALID;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int m = std::min(knn_m, N - 1);
  prof_begin(RIFT_PROF_SCORE, st);
  const int nk = launch_smooth(V, tile_s_raw, N, d, row0, n_rows, m, tile_s, nbr, static_cast<char*>(ws), st);
  prof_end(RIFT_PROF_SCORE, st, nk < 0 ? 0 : nk);
  if (nk < 0) return RIFT_ERR_CUDA;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

rift_status rift_score_range(const float* tile_s, int n, float* range, rift_stream_t stream) {
  if (!tile_s || !range || n < 1 || n > RIFT_MAX_TILES) return RIFT_ERR_INVALID;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  prof_begin(RIFT_PROF_SELECT, st);
  launch_score_range(tile_s, n, range, st);
  prof_end(RIFT_PROF_SELECT, st, 1);
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

rift_status rift_select_budgeted_tokens_ranged(const float* token_scores, const float* tile_s, int N, int n_v,
                                               const float* s_range, const float* p, const rift_policy* policy,
                                               float* u, int* kept, int* n_kept, int* budgets, int* sel,
                                               int* sel_off, rift_stream_t stream) {
  if (!s_range) return RIFT_ERR_INVALID;
  const rift_status chk =
      select_args_check(token_scores, tile_s, N, n_v, policy, u, kept, n_kept, budgets, sel, sel_off);
  if (chk != RIFT_OK) return chk;
  prof_begin(RIFT_PROF_SELECT, static_cast<cudaStream_t>(stream));
  const int launches = launch_select(token_scores, tile_s, N, n_v, p, *policy, u, kept, n_kept, budgets, sel, sel_off,
                                     static_cast<cudaStream_t>(stream), s_range);
  prof_end(RIFT_PROF_SELECT, static_cast<cudaStream_t>(stream), launches);
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

rift_status rift_pack_ragged(const void* X, rift_dtype xdt, int N, int n_v, int d, const int* kept,
                             const int* n_kept, const int* sel, const int* sel_off, const int* sys_ids, int S,
                             const int* query_ids, int Q, const void* embed, int vocab, const void* ctx,
                             const int* ctx_off, void* packed, int max_T, int* cu_seqlens, int* positions, int* T,
                             rift_stream_t stream) {
  return rift_pack_ragged_at(X, xdt, N, n_v, d, kept, n_kept, sel, sel_off, sys_ids, S, query_ids, Q, embed, vocab,
                             ctx, ctx_off, packed, max_T, cu_seqlens, positions, T, 0, stream);
}

rift_status rift_pack_ragged_at(const void* X, rift_dtype xdt, int N, int n_v, int d, const int* kept,
                                const int* n_kept, const int* sel, const int* sel_off, const int* sys_ids, int S,
                                const int* query_ids, int Q, const void* embed, int vocab, const void* ctx,
                                const int* ctx_off, void* packed, int max_T, int* cu_seqlens, int* positions,
                                int* T, int row_base, rift_stream_t stream) {
  if (!dims_ok(N, n_v, d) || !X || !kept || !n_kept || !sel || !sel_off || !embed || !packed || !cu_seqlens ||
      !positions || !T || row_base < 0)
    return RIFT_ERR_INVALID;
  if (xdt != RIFT_F32 && xdt != RIFT_BF16) return RIFT_ERR_INVALID;
  if (S < 0 || Q < 0 || (S > 0 && !sys_ids) || (Q > 0 && !query_ids) || vocab < 1 || max_T < 0)
    return RIFT_ERR_INVALID;
  if (!aligned16(X) || !aligned16(embed) || !aligned16(packed)) return RIFT_ERR_INVALID;
  if ((ctx == nullptr) != (ctx_off == nullptr) || (ctx && !aligned16(ctx))) return RIFT_ERR_INVALID;
  prof_begin(RIFT_PROF_PACK, static_cast<cudaStream_t>(stream));
  launch_pack(X, xdt, N, n_v, d, kept, n_kept, sel, sel_off, sys_ids, S, query_ids, Q, embed, vocab, ctx, ctx_off,
              packed, max_T, cu_seqlens, positions, T, row_base, static_cast<cudaStream_t>(stream));
  prof_end(RIFT_PROF_PACK, static_cast<cudaStream_t>(stream), 2);
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_features_workspace_bytes(int N, int d) {
  if (N < 1 || N > RIFT_MAX_TILES || d < 64 || d > 8192 || d % 64 != 0) return 0;
  return features_layout(N, d).total;
}

rift_status rift_tile_features(const void* X, rift_dtype xdt, int N, int n_v, int d, const float* t, const float* B,
                               int M, const float* token_scores, const int* tiles, const int* n_tiles,
                               float* features, float* V, void* ws, size_t ws_bytes, rift_stream_t stream) {
  if (!dims_ok(N, n_v, d) || !X || !t || !token_scores || !features) return RIFT_ERR_INVALID;
  if (xdt != RIFT_F32 && xdt != RIFT_BF16) return RIFT_ERR_INVALID;
  if (M < 0 || M > 64 || (M > 0 && !B) || (tiles == nullptr) != (n_tiles == nullptr)) return RIFT_ERR_INVALID;
  if (!aligned16(X) || !aligned16(features) || (V && !aligned16(V))) return RIFT_ERR_INVALID;
  if (!ws_ok(ws, ws_bytes, features_layout(N, d).total)) return RIFT_ERR_INVALID;
  int g = 0;
  while ((g + 1) * (g + 1) <= n_v) ++g;
  if (g * g != n_v || g % 2 != 0) return RIFT_ERR_UNSUPPORTED;
  prof_begin(RIFT_PROF_SCORE, static_cast<cudaStream_t>(stream));
  const int nk = launch_features(X, xdt, N, n_v, d, g, t, B, M, token_scores, tiles, n_tiles, features, V,
                                 static_cast<char*>(ws), static_cast<cudaStream_t>(stream));
  prof_end(RIFT_PROF_SCORE, static_cast<cudaStream_t>(stream), nk);
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_merge_workspace_bytes(int N, int n_v) {
  if (N < 1 || N > RIFT_MAX_TILES || n_v < 1 || n_v > RIFT_MAX_NV) return 0;
  return merge_layout(N, n_v).total;
}

rift_status rift_merge_contextual(const void* X, rift_dtype xdt, int N, int n_v, int d, const int* kept,
                                  const int* n_kept, const int* budgets, const int* sel, const int* sel_off, void* ctx,
                                  int max_ctx, int* ctx_off, int* ctx_target, void* ws, size_t ws_bytes,
                                  rift_stream_t stream) {
  if (!dims_ok(N, n_v, d) || !X || !kept || !n_kept || !budgets || !sel || !sel_off || !ctx_off || !ctx_target ||
      max_ctx < 0 || (max_ctx > 0 && !ctx))
    return RIFT_ERR_INVALID;
  if (xdt != RIFT_F32 && xdt != RIFT_BF16) return RIFT_ERR_INVALID;
  if (!aligned16(X) || (ctx && !aligned16(ctx))) return RIFT_ERR_INVALID;
  if (!ws_ok(ws, ws_bytes, merge_layout(N, n_v).total)) return RIFT_ERR_INVALID;
  prof_begin(RIFT_PROF_SELECT, static_cast<cudaStream_t>(stream));
  const int nk = launch_merge(X, xdt, N, n_v, d, kept, n_kept, budgets, sel, sel_off, static_cast<uint16_t*>(ctx),
                              max_ctx, ctx_off, ctx_target, static_cast<char*>(ws), static_cast<cudaStream_t>(stream));
  if (nk < 0) return RIFT_ERR_CUDA;
  prof_end(RIFT_PROF_SELECT, static_cast<cudaStream_t>(stream), nk);
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

static bool model_ok(const rift_model* m) {
  if (!m) return false;
  if (m->n_layers < 1 || m->d < 64 || m->d > 8192 || m->d % 64 != 0) return false;
  if (m->head_dim != 64 && m->head_dim != 128) return false;
  if (m->n_heads < 1 || m->n_heads * m->head_dim != m->d) return false;
  if (m->ffn < 16 || m->ffn % 16 != 0) return false;
  if (!(m->eps > 0.f) || !(m->rope_theta > 0.f)) return false;
  if (!m->w_qkv || !m->w_o || !m->w_gate_up || !m->w_down || !m->g_attn || !m->g_ffn || !m->g_final)
    return false;
  for (int l = 0; l < m->n_layers; ++l) {
    const void* p[6] = {m->w_qkv[l], m->w_o[l], m->w_gate_up[l], m->w_down[l], m->g_attn[l], m->g_ffn[l]};
    for (const void* q : p)
      if (!q || !aligned16(q)) return false;
  }
  return aligned16(m->g_final);
}

rift_status rift_check_wait_timeout(rift_stream_t stream) {
  launch_wait_timeout_check(static_cast<cudaStream_t>(stream));
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_prefill_workspace_bytes(const rift_model* m, int max_T, int max_seqs, int max_len) {
  if (!model_ok(m) || max_T < 0 || max_seqs < 0 || max_len < 1) return 0;
  return prefill_layout(*m, max_T, max_seqs, max_len).total;
}

static bool lm_head_ok(const rift_model* m) {
  return m->lm_head && aligned16(m->lm_head) && m->vocab >= 8 && m->vocab % 8 == 0;
}

rift_status rift_prefill_layers(const rift_model* m, void* hidden, const int* T, int max_T, const int* cu_seqlens,
                                const int* n_seq, int max_seqs, int max_len, const int* positions, void* kv_out,
                                float* last_logits, void* ws, size_t ws_bytes, rift_stream_t stream) {
  if (!model_ok(m) || !hidden || !cu_seqlens || !positions || max_T < 0 || max_seqs < 0 || max_len < 1)
    return RIFT_ERR_INVALID;
  if (max_T > 0 && max_seqs < 1) return RIFT_ERR_INVALID;
  if (!aligned16(hidden) || (kv_out && !aligned16(kv_out)) || (last_logits && !aligned16(last_logits)))
    return RIFT_ERR_INVALID;
  if (last_logits && !lm_head_ok(m)) return RIFT_ERR_INVALID;
  const size_t need = prefill_layout(*m, max_T, max_seqs, max_len).total;
  if (!ws_ok(ws, ws_bytes, need)) return RIFT_ERR_INVALID;
  if (launch_prefill(*m, hidden, max_T, T, cu_seqlens, max_seqs, n_seq, max_len, positions, kv_out, last_logits,
                     static_cast<char*>(ws), static_cast<cudaStream_t>(stream)))
    return RIFT_ERR_INVALID;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_prefill_shared_prefix_workspace_bytes(const rift_model* m, int max_T, int max_seqs, int max_len, int S) {
  if (!model_ok(m) || max_T < 0 || max_seqs < 0 || max_len < 1 || S < 1 || S > max_len) return 0;
  return shared_prefix_layout(*m, max_T, max_seqs, max_len, S).total;
}

rift_status rift_prefill_shared_prefix(const rift_model* m, const int* sys_ids, int S, const void* embed, int vocab,
                                       void* prefix_hidden, void* prefix_kv, void* hidden, const int* T, int max_T,
                                       const int* cu_seqlens, const int* n_seq, int max_seqs, int max_len,
                                       const int* positions, float* last_logits, void* ws, size_t ws_bytes,
                                       rift_stream_t stream) {
  if (!model_ok(m) || !sys_ids || !embed || !prefix_hidden || !prefix_kv || S < 1 || vocab < 1 || max_T < 0 ||
      max_seqs < 0 || max_len < 1 || S > max_len)
    return RIFT_ERR_INVALID;
  if (max_T > 0 && (!hidden || !cu_seqlens || !positions || max_seqs < 1)) return RIFT_ERR_INVALID;
  if (!aligned16(embed) || !aligned16(prefix_hidden) || !aligned16(prefix_kv) || (hidden && !aligned16(hidden)) ||
      (last_logits && !aligned16(last_logits)))
    return RIFT_ERR_INVALID;
  if (last_logits && !lm_head_ok(m)) return RIFT_ERR_INVALID;
  if (!ws_ok(ws, ws_bytes, shared_prefix_layout(*m, max_T, max_seqs, max_len, S).total)) return RIFT_ERR_INVALID;
  if (launch_prefill_shared_prefix(*m, sys_ids, S, embed, vocab, prefix_hidden, prefix_kv, hidden, max_T, T,
                                   cu_seqlens, max_seqs, n_seq, max_len, positions, last_logits,
                                   static_cast<char*>(ws), static_cast<cudaStream_t>(stream)))
    return RIFT_ERR_INVALID;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_decode_workspace_bytes(const rift_model* m, int n_seq, int max_len) {
  if (!model_ok(m) || n_seq < 0 || max_len < 1 || max_len > 32768) return 0;
  return decode_layout(*m, n_seq, max_len).total;
}

rift_status rift_decode_step(const rift_model* m, const void* kv_cache, int T, const int* cu_seqlens, int n_seq,
                             int max_len, const int* token_ids, const void* embed, int vocab_embed,
                             void* hidden_out, void* kv_new, float* logits, void* ws, size_t ws_bytes,
                             rift_stream_t stream) {
  if (!model_ok(m) || !kv_cache || !cu_seqlens || !token_ids || !embed || T < 0 || n_seq < 0 || max_len < 1 ||
      max_len > 32768 || vocab_embed < 1)
    return RIFT_ERR_INVALID;
  if (!aligned16(kv_cache) || !aligned16(embed) || (hidden_out && !aligned16(hidden_out)) ||
      (kv_new && !aligned16(kv_new)) || (logits && !aligned16(logits)))
    return RIFT_ERR_INVALID;
  if (logits && !lm_head_ok(m)) return RIFT_ERR_INVALID;
  const size_t need = decode_layout(*m, n_seq, max_len).total;
  if (!ws_ok(ws, ws_bytes, need)) return RIFT_ERR_INVALID;
  if (launch_decode(*m, kv_cache, T, cu_seqlens, n_seq, max_len, token_ids, embed, vocab_embed, hidden_out, kv_new,
                    logits, static_cast<char*>(ws), static_cast<cudaStream_t>(stream)))
    return RIFT_ERR_INVALID;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

rift_status rift_linear(const void* A, const void* W, int M, int N, int K, int epilogue, void* out,
                        rift_stream_t stream) {
  if (!A || !W || !out || M < 0 || N < 1 || K < 1) return RIFT_ERR_INVALID;
  if (epilogue < RIFT_EPI_STORE_F16 || epilogue > RIFT_EPI_SWIGLU) return RIFT_ERR_INVALID;
  if (K % 8 != 0 || N % 8 != 0 || (epilogue == RIFT_EPI_SWIGLU && N % 32 != 0)) return RIFT_ERR_INVALID;
  if (!aligned16(A) || !aligned16(W) || !aligned16(out)) return RIFT_ERR_INVALID;
  if (M == 0) return RIFT_OK;
  if (launch_gemm(A, W, M, N, K, epilogue, out, static_cast<cudaStream_t>(stream))) return RIFT_ERR_CUDA;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_attention_workspace_bytes(int max_T, int max_seqs) {
  if (max_T <= 0 || max_seqs < 0) return 0;  // no rows: nothing to schedule
  return (size_t)(attention_max_qblocks(max_T, max_seqs) + 1) * sizeof(int4);
}

rift_status rift_attention_varlen(const void* qkv, int T, const int* cu_seqlens, int n_seq, int n_heads,
                                  int head_dim, void* out, void* ws, size_t ws_bytes, rift_stream_t stream) {
  if (!qkv || !cu_seqlens || !out || T < 0 || n_seq < 0 || n_heads < 1) return RIFT_ERR_INVALID;
  if (head_dim != 64 && head_dim != 128) return RIFT_ERR_INVALID;
  if (T > 0 && n_seq < 1) return RIFT_ERR_INVALID;
  if (!aligned16(qkv) || !aligned16(out)) return RIFT_ERR_INVALID;
  const size_t need = rift_attention_workspace_bytes(T, n_seq);
  if (!ws_ok(ws, ws_bytes, need)) return RIFT_ERR_INVALID;
  if (T == 0) return RIFT_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int4* sched = static_cast<int4*>(ws);
  const int n_max = attention_max_qblocks(T, n_seq);
  prof_begin(RIFT_PROF_ATTN, st);
  launch_attention_schedule(cu_seqlens, n_seq, nullptr, T, sched, n_max, st);
  if (launch_attention(qkv, T, cu_seqlens, n_seq, n_heads, head_dim, sched, n_max, out, st)) return RIFT_ERR_CUDA;
  prof_end(RIFT_PROF_ATTN, st, 2);
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

// ---- rotary positions, the paged cache ----

static bool in_type(rift_dtype dt) { return dt == RIFT_F32 || dt == RIFT_F16 || dt == RIFT_BF16; }
static int type_size(rift_dtype dt) { return dt == RIFT_F32 ? 4 : dt == RIFT_E4M3 ? 1 : 2; }

// Rows of `width` elements `stride` apart that may be read and written 16 bytes at a time.
static bool rows_ok(const void* p, long long stride, long long width, rift_dtype dt) {
  return p && aligned16(p) && stride >= width && stride <= 0x7fffffffLL && stride * type_size(dt) % 16 == 0;
}

// Whether n_rows rows of a_width elements at a and of b_width at b share no memory.
static bool apart(const void* a, long long a_stride, long long a_width, const void* b, long long b_stride, long long b_width,
                  long long n_rows, rift_dtype dt) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  const int size = type_size(dt);
  if (x + ((n_rows - 1) * a_stride + a_width) * size <= y || y + ((n_rows - 1) * b_stride + b_width) * size <= x) return true;
  // slices of the same rows (columns of one buffer)
  if (a_stride != b_stride) return false;
  const uintptr_t pitch = a_stride * size, off = (x > y ? x - y : y - x) % pitch;
  const long long low = x < y ? a_width : b_width, high = x < y ? b_width : a_width;
  return off >= (uintptr_t)(low * size) && off + high * size <= pitch;
}
// ... or, of one width, are the same rows.
static bool apart_or_same(const void* a, long long a_stride, const void* b, long long b_stride, long long n_rows,
                          long long width, rift_dtype dt) {
  return (a == b && a_stride == b_stride) || apart(a, a_stride, width, b, b_stride, width, n_rows, dt);
}

static bool positive(double x) { return std::isfinite(x) && x > 0.0; }

static bool spec_ok(const rift_rope_spec* s, int head_dim) {
  if (!s || s->rot_dim < 2 || s->rot_dim % 2 != 0 || s->rot_dim > head_dim) return false;
  if (!positive(s->theta) || !positive(s->amplitude) || s->amplitude > 1e30) return false;
  if (s->scaling < RIFT_ROPE_PLAIN || s->scaling > RIFT_ROPE_PARTS) return false;
  if (s->scaling != RIFT_ROPE_PLAIN && !positive(s->factor)) return false;
  if (s->scaling == RIFT_ROPE_PARTS &&
      !(positive(s->orig_len) && std::isfinite(s->high) && s->low >= 0.0 && s->low < s->high))
    return false;
  return true;
}

rift_status rift_rope(const void* x, rift_dtype dt, int T, int n_heads, int head_dim, long long x_stride,
                      const int* positions, const rift_rope_spec* spec, int inverse, void* out, long long out_stride,
                      rift_stream_t stream) {
  if (!in_type(dt) || T < 0 || n_heads < 1 || n_heads > 65536 || head_dim < 2 || head_dim % 2 != 0 ||
      head_dim > RIFT_ROPE_MAX_HEAD_DIM || !spec_ok(spec, head_dim))
    return RIFT_ERR_INVALID;
  if (T == 0) return RIFT_OK;
  const long long width = (long long)n_heads * head_dim;
  if (!x || !out || !positions || !aligned16(x) || !aligned16(out) || x_stride < width || out_stride < width ||
      x_stride > 0x7fffffffLL || out_stride > 0x7fffffffLL)
    return RIFT_ERR_INVALID;
  if (!apart_or_same(x, x_stride, out, out_stride, T, width, dt)) return RIFT_ERR_INVALID;
  const RopeAngles R = rope_angles(*spec, inverse != 0);
  if (!R.ok) return RIFT_ERR_INVALID;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  prof_begin(RIFT_PROF_ROPE, st);
  const bool ok = launch_rope(x, dt, T, n_heads, head_dim, x_stride, positions, R, out, out_stride, st);
  prof_end(RIFT_PROF_ROPE, st, ok ? 1 : 0);
  if (!ok) return RIFT_ERR_CUDA;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

// The pool's description checked, and as the kernels take it.
static bool pool_of(const rift_kv_pages* c, KvPool* P) {
  if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return false;
  if (c->dtype != RIFT_F16 && c->dtype != RIFT_BF16 && c->dtype != RIFT_E4M3) return false;
  if ((c->dtype == RIFT_E4M3) != (c->k_scale != nullptr) || (c->dtype == RIFT_E4M3) != (c->v_scale != nullptr)) return false;
  if (c->n_pages < 1 || c->page_size < 1 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0) return false;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 4096 || (c->head_dim != 64 && c->head_dim != 128)) return false;
  const long long most = 1LL << 40, hd = c->head_dim, n = c->n_kv_heads, ps = c->page_size;
  for (long long s : {c->page_stride, c->row_stride, c->head_stride})
    if (s < 0 || s > most || s * type_size(c->dtype) % 16 != 0) return false;
  if (c->row_stride > 0x7fffffffLL || c->head_stride > 0x7fffffffLL) return false;
  // a row's heads apart and rows apart from each other (or a head's rows, and heads), pages apart
  const bool rows_of_heads = (n == 1 || c->head_stride >= hd) && (ps == 1 || c->row_stride >= (n - 1) * c->head_stride + hd);
  const bool heads_of_rows = (ps == 1 || c->row_stride >= hd) && (n == 1 || c->head_stride >= (ps - 1) * c->row_stride + hd);
  if (!rows_of_heads && !heads_of_rows) return false;
  // a row's offset in units of the largest power of two (up to 2^20 bytes) that divides the strides has to fit 32 bits
  const long long es = type_size(c->dtype), strides = (c->page_stride | c->row_stride | c->head_stride) * es;
  long long unit = 16;
  while (unit < (1 << 20) && strides % (2 * unit) == 0) unit *= 2;
  const __int128 furthest = (__int128)(c->n_pages - 1) * c->page_stride + (ps - 1) * c->row_stride + (n - 1) * c->head_stride;
  if (furthest * es / unit >= (1LL << 32)) return false;
  if (c->n_pages > 1 && c->page_stride < (ps - 1) * c->row_stride + (n - 1) * c->head_stride + hd) return false;
  int shift = 0;
  while ((1 << shift) < c->page_size) ++shift;
  *P = KvPool{c->k, c->v, c->k_scale, c->v_scale, c->n_pages, shift, c->n_kv_heads, c->head_dim,
              c->page_stride, (int)c->row_stride, (int)c->head_stride};
  return true;
}

// Whether a table of max_pages pages has positions that fit an int, with room for a tile behind the last.
static bool table_ok(int max_pages, int ps_shift) {
  return max_pages >= 1 && ((long long)max_pages << ps_shift) <= RIFT_MAX_POSITIONS;
}

// The rows of a call and their sequences (a call without rows needs no arrays: they may be empty tensors).
static bool rows_args_ok(int T, const int* cu_seqlens, const int* start, int n_seq, const int* page_table, int max_pages,
                         int ps_shift) {
  if (T < 0 || n_seq < 0 || !table_ok(max_pages, ps_shift) || (!cu_seqlens && T != n_seq)) return false;
  return T == 0 || n_seq == 0 || (start && page_table);
}

rift_status rift_kv_append(const rift_kv_pages* cache, const void* k, long long k_stride, const void* v,
                           long long v_stride, rift_dtype dt, int T, const int* cu_seqlens, const int* start, int n_seq,
                           const int* page_table, int max_pages, const rift_rope_spec* rope, const void* q,
                           long long q_stride, int n_q_heads, void* q_out, long long q_out_stride, rift_stream_t stream) {
  KvPool P;
  if (!pool_of(cache, &P) || !in_type(dt) || !rows_args_ok(T, cu_seqlens, start, n_seq, page_table, max_pages, P.ps_shift))
    return RIFT_ERR_INVALID;
  if (rope && !spec_ok(rope, P.head_dim)) return RIFT_ERR_INVALID;
  if (T == 0 || n_seq == 0) return RIFT_OK;
  const long long width = (long long)P.n_kv * P.head_dim;
  if (!rows_ok(k, k_stride, width, dt) || !rows_ok(v, v_stride, width, dt)) return RIFT_ERR_INVALID;
  if ((q == nullptr) != (q_out == nullptr) || (q && !rope)) return RIFT_ERR_INVALID;
  if (q) {
    if (n_q_heads < 1 || n_q_heads > 65536) return RIFT_ERR_INVALID;
    const long long qw = (long long)n_q_heads * P.head_dim;
    if (!rows_ok(q, q_stride, qw, dt) || !rows_ok(q_out, q_out_stride, qw, dt)) return RIFT_ERR_INVALID;
    if (!apart_or_same(q, q_stride, q_out, q_out_stride, T, qw, dt)) return RIFT_ERR_INVALID;
    if (!apart(q_out, q_out_stride, qw, k, k_stride, width, T, dt) || !apart(q_out, q_out_stride, qw, v, v_stride, width, T, dt))
      return RIFT_ERR_INVALID;
  }
  if (rope && rope->rot_dim % 16 != 0) return RIFT_ERR_UNSUPPORTED;
  RopeAngles R;
  if (rope) {
    R = rope_angles(*rope, false);
    if (!R.ok) return RIFT_ERR_INVALID;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  g_paged_used = true;
  prof_begin(RIFT_PROF_PACK, st);
  const bool ok = launch_kv_append(P, cache->dtype, k, k_stride, v, v_stride, dt, T, cu_seqlens, start, n_seq, page_table, max_pages,
                   rope ? &R : nullptr, q, q_stride, q ? n_q_heads : 0, q_out, q_out_stride, st);
  prof_end(RIFT_PROF_PACK, st, ok ? 1 : 0);
  if (!ok) return RIFT_ERR_CUDA;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

rift_status rift_kv_gather(const rift_kv_pages* cache, int T, const int* cu_seqlens, const int* start, int n_seq,
                           const int* page_table, int max_pages, void* k, long long k_stride, void* v,
                           long long v_stride, rift_dtype dt, rift_stream_t stream) {
  KvPool P;
  if (!pool_of(cache, &P) || !in_type(dt) || !rows_args_ok(T, cu_seqlens, start, n_seq, page_table, max_pages, P.ps_shift))
    return RIFT_ERR_INVALID;
  if (T == 0 || n_seq == 0) return RIFT_OK;
  const long long width = (long long)P.n_kv * P.head_dim;
  if ((!k && !v) || (k && !rows_ok(k, k_stride, width, dt)) || (v && !rows_ok(v, v_stride, width, dt)))
    return RIFT_ERR_INVALID;
  if (k && v && !apart(k, k_stride, width, v, v_stride, width, T, dt)) return RIFT_ERR_INVALID;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  g_paged_used = true;
  prof_begin(RIFT_PROF_PACK, st);
  const bool ok = launch_kv_gather(P, cache->dtype, T, cu_seqlens, start, n_seq, page_table, max_pages, k, k_stride, v, v_stride, dt, st);
  prof_end(RIFT_PROF_PACK, st, ok ? 1 : 0);
  if (!ok) return RIFT_ERR_CUDA;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

static bool paged_dims_ok(int n_seq, int n_heads, int n_kv, int head_dim) {
  return n_seq >= 0 && n_kv >= 1 && n_kv <= 4096 && n_heads >= 1 && n_heads <= 65536 && n_heads % n_kv == 0 &&
         (long long)n_seq * n_heads <= (1LL << 28) && (head_dim == 64 || head_dim == 128);
}

size_t rift_attention_paged_workspace_bytes(int n_seq, int n_heads, int n_kv_heads, int head_dim) {
  if (!paged_dims_ok(n_seq, n_heads, n_kv_heads, head_dim) || n_seq == 0) return 0;
  return paged_attention_workspace(n_seq, n_heads, n_kv_heads, head_dim);
}

rift_status rift_attention_paged(const rift_kv_pages* cache, const void* q, rift_dtype dt, long long q_stride,
                                 int n_heads, const int* seq_lens, int n_seq, const int* page_table, int max_pages,
                                 int window, float scale, void* out, long long out_stride, float* lse, void* ws,
                                 size_t ws_bytes, rift_stream_t stream) {
  KvPool P;
  if (!pool_of(cache, &P) || !paged_dims_ok(n_seq, n_heads, P.n_kv, P.head_dim)) return RIFT_ERR_INVALID;
  if ((dt != RIFT_F16 && dt != RIFT_BF16) || !table_ok(max_pages, P.ps_shift) || window < 0) return RIFT_ERR_INVALID;
  if (cache->dtype != RIFT_E4M3 && cache->dtype != dt) return RIFT_ERR_INVALID;
  if (!std::isfinite(scale) || scale < 0.f) return RIFT_ERR_INVALID;
  if (n_seq == 0) return RIFT_OK;
  if (!seq_lens || !page_table) return RIFT_ERR_INVALID;
  const long long width = (long long)n_heads * P.head_dim;
  if (!rows_ok(q, q_stride, width, dt) || !rows_ok(out, out_stride, width, dt)) return RIFT_ERR_INVALID;
  if (!apart_or_same(q, q_stride, out, out_stride, n_seq, width, dt)) return RIFT_ERR_INVALID;
  if (!ws_ok(ws, ws_bytes, rift_attention_paged_workspace_bytes(n_seq, n_heads, P.n_kv, P.head_dim))) return RIFT_ERR_INVALID;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  g_paged_used = true;
  prof_begin(RIFT_PROF_ATTN, st);
  const int nk = launch_attention_paged(P, cache->dtype, q, dt, q_stride, n_heads, seq_lens, n_seq, page_table, max_pages,
                                        window, scale > 0.f ? scale : 1.f / std::sqrt((float)P.head_dim), out, out_stride,
                                        lse, static_cast<char*>(ws), st);
  prof_end(RIFT_PROF_ATTN, st, nk < 0 ? 0 : nk);
  if (nk < 0) return RIFT_ERR_CUDA;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

size_t rift_decode_paged_workspace_bytes(const rift_model* m, int n_seq) {
  if (!model_ok(m) || n_seq < 0 || !paged_dims_ok(n_seq, m->n_heads, m->n_heads, m->head_dim)) return 0;
  return decode_paged_layout(*m, n_seq).total;
}

rift_status rift_decode_step_paged(const rift_model* m, const rift_kv_pages* cache, const int* page_table,
                                   int max_pages, const int* seq_lens, int n_seq, const int* token_ids,
                                   const void* embed, int vocab_embed, void* hidden_out, float* logits, void* ws,
                                   size_t ws_bytes, rift_stream_t stream) {
  if (!model_ok(m) || !cache || !page_table || !seq_lens || !token_ids || !embed || n_seq < 0 || max_pages < 1 ||
      vocab_embed < 1 || !paged_dims_ok(n_seq, m->n_heads, m->n_heads, m->head_dim))
    return RIFT_ERR_INVALID;
  if (!aligned16(embed) || (hidden_out && !aligned16(hidden_out)) || (logits && !aligned16(logits))) return RIFT_ERR_INVALID;
  if (logits && !lm_head_ok(m)) return RIFT_ERR_INVALID;
  if (m->n_layers > 1024) return RIFT_ERR_UNSUPPORTED;
  KvPool pools[1024];
  for (int l = 0; l < m->n_layers; ++l) {
    if (!pool_of(&cache[l], &pools[l]) || cache[l].dtype == RIFT_BF16 || cache[l].n_kv_heads != m->n_heads ||
        cache[l].head_dim != m->head_dim || cache[l].page_size != cache[0].page_size)
      return RIFT_ERR_INVALID;
  }
  const long long capacity = (long long)max_pages * cache[0].page_size;
  if (!table_ok(max_pages, pools[0].ps_shift)) return RIFT_ERR_INVALID;
  if (!ws_ok(ws, ws_bytes, decode_paged_layout(*m, n_seq).total)) return RIFT_ERR_INVALID;
  if (n_seq == 0) return RIFT_OK;
  g_paged_used = true;
  if (launch_decode_paged(*m, cache, pools, page_table, max_pages, (int)capacity, seq_lens, n_seq, token_ids, embed,
                          vocab_embed, hidden_out, logits, static_cast<char*>(ws), static_cast<cudaStream_t>(stream)))
    return RIFT_ERR_CUDA;
  RIFT_LAUNCH_CHECK();
  return RIFT_OK;
}

}  // extern "C"
