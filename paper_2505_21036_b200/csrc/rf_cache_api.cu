// C ABI of the paged 8-bit K/V cache: argument validation and hand-over to the launchers.
#include <math.h>

#include "rf_cache.cuh"

namespace {

bool aligned(const void* p, uintptr_t n) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

rf_status check_cache(const rf_cache* c, RfCache* out) {
  if (c == nullptr) return RF_ERR_INVALID_ARG;
  if (c->n_seqs < 1 || c->heads < 1 || c->n_pages < 1 || c->max_pages < 1) return RF_ERR_INVALID_ARG;
  if (c->D != 64 && c->D != 96 && c->D != 128) return c->D < 1 ? RF_ERR_INVALID_ARG : RF_ERR_UNSUPPORTED;
  if (c->n_seqs > kCacheMaxSeqs || (long long)c->n_seqs * c->heads > 65535 || c->n_pages > kCacheMaxPages || c->max_pages > (1 << 23) ||
      (long long)c->n_pages * c->heads > 0x7fffffffll)
    return RF_ERR_UNSUPPORTED;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_sum, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4) ||
      !aligned(c->page_table, 4) || !aligned(c->seq_len, 4))
    return RF_ERR_INVALID_ARG;
  *out = RfCache{c->n_seqs, c->heads, c->D, c->n_pages, c->max_pages, c->k, c->v, c->k_scale, c->v_scale, c->k_sum, c->page_table, c->seq_len};
  return RF_OK;
}

rf_status check_query(const RfCache& c, const rf_cache_query* u, RfQueries* out) {
  if (u == nullptr || u->H < 1 || u->M < 1 || u->causal_block < 0 || !(u->scale >= 0.f && isfinite(u->scale)) || u->H % c.H != 0) return RF_ERR_INVALID_ARG;
  const long long rows = (long long)(u->H / c.H) * u->M;
  if (rows > (1ll << 30) || (long long)c.B * c.H * ((rows + 15) / 16) > (1ll << 30)) return RF_ERR_UNSUPPORTED;
  *out = RfQueries{u->M, u->H / c.H, (int)rows, (int)((rows + kPage - 1) / kPage), u->causal_block, nullptr, nullptr, nullptr};
  return RF_OK;
}

rf_status check_ws(const void* ws, size_t have, size_t need) {
  if (!aligned(ws, 256)) return RF_ERR_INVALID_ARG;
  return have < need ? RF_ERR_WORKSPACE_TOO_SMALL : RF_OK;
}

rf_status done(cudaError_t e) { return e == cudaSuccess ? RF_OK : RF_ERR_CUDA; }

}  // namespace

extern "C" {

size_t rf_cache_workspace_bytes(const rf_cache* cache) {
  RfCache c;
  return check_cache(cache, &c) == RF_OK ? rf_cache_ws_words(c) * sizeof(int32_t) : 0;
}

rf_status rf_cache_append(const rf_cache* cache, const void* k, const void* v, int32_t M, const int32_t* new_len, void* ws,
                          size_t ws_bytes, int32_t* dev_status, void* cuda_stream) {
  RfCache c;
  rf_status st = check_cache(cache, &c);
  if (st != RF_OK) return st;
  if (!aligned(k, 16) || !aligned(v, 16) || M < 1) return RF_ERR_INVALID_ARG;
  if (M > (1 << 30)) return RF_ERR_UNSUPPORTED;
  st = check_ws(ws, ws_bytes, rf_cache_ws_words(c) * sizeof(int32_t));
  if (st != RF_OK) return st;
  return done(rf_launch_cache_append(c, static_cast<const __nv_bfloat16*>(k), static_cast<const __nv_bfloat16*>(v), M, new_len,
                                     static_cast<int32_t*>(ws), dev_status, static_cast<cudaStream_t>(cuda_stream)));
}

rf_status rf_cache_fork(const rf_cache* cache, const int32_t* parent, int32_t* dev_status, void* cuda_stream) {
  RfCache c;
  const rf_status st = check_cache(cache, &c);
  if (st != RF_OK) return st;
  if (parent == nullptr) return RF_ERR_INVALID_ARG;
  return done(rf_launch_cache_fork(c, parent, dev_status, static_cast<cudaStream_t>(cuda_stream)));
}

rf_status rf_cache_drop(const rf_cache* cache, const int32_t* first, const int32_t* count, const int32_t* max_len, int32_t* dev_status,
                        void* cuda_stream) {
  RfCache c;
  const rf_status st = check_cache(cache, &c);
  if (st != RF_OK) return st;
  if ((first == nullptr) != (count == nullptr) || (first == nullptr && max_len == nullptr)) return RF_ERR_INVALID_ARG;
  return done(rf_launch_cache_drop(c, first, count, max_len, dev_status, static_cast<cudaStream_t>(cuda_stream)));
}

rf_status rf_cache_compact(const rf_cache* cache, int32_t* n_live, void* ws, size_t ws_bytes, int32_t* dev_status, void* cuda_stream) {
  RfCache c;
  rf_status st = check_cache(cache, &c);
  if (st != RF_OK) return st;
  if (n_live == nullptr) return RF_ERR_INVALID_ARG;
  st = check_ws(ws, ws_bytes, rf_cache_ws_words(c) * sizeof(int32_t));
  if (st != RF_OK) return st;
  return done(rf_launch_cache_compact(c, n_live, static_cast<int32_t*>(ws), dev_status, static_cast<cudaStream_t>(cuda_stream)));
}

rf_status rf_cache_select(const rf_cache* cache, const rf_cache_query* query, const void* q, const int32_t* q_len, int32_t keep_first,
                          int32_t keep_last, int32_t top_k, rf_schedule* out, int32_t* dev_status, void* cuda_stream) {
  return rf_cache_select_origin(cache, query, q, q_len, nullptr, keep_first, keep_last, top_k, out, dev_status, cuda_stream);
}

rf_status rf_cache_select_origin(const rf_cache* cache, const rf_cache_query* query, const void* q, const int32_t* q_len,
                                 const int32_t* block_origin, int32_t keep_first, int32_t keep_last, int32_t top_k, rf_schedule* out,
                                 int32_t* dev_status, void* cuda_stream) {
  RfCache c;
  RfQueries u;
  rf_status st = check_cache(cache, &c);
  if (st == RF_OK) st = check_query(c, query, &u);
  if (st != RF_OK) return st;
  if (!aligned(q, 16) || out == nullptr || out->count == nullptr || out->kv_tile == nullptr) return RF_ERR_INVALID_ARG;
  if (keep_first < 0 || keep_last < 0 || top_k < 0 || out->nQ != u.n_q || out->nKmax < 1) return RF_ERR_INVALID_ARG;
  const long long wanted = (long long)keep_first + keep_last + top_k;
  if (out->nKmax < (wanted < c.max_pages ? wanted : c.max_pages)) return RF_ERR_INVALID_ARG;
  if (c.max_pages > kSelectMaxPages) return RF_ERR_UNSUPPORTED;
  u.q = static_cast<const __nv_bfloat16*>(q);
  u.q_len = q_len;
  u.origin = block_origin;
  return done(rf_launch_cache_select(c, u, keep_first, keep_last, top_k, out->count, out->kv_tile, out->nKmax, dev_status,
                                     static_cast<cudaStream_t>(cuda_stream)));
}

size_t rf_cache_attn_workspace_bytes(const rf_cache* cache, const rf_cache_query* query) {
  RfCache c;
  RfQueries u;
  return check_cache(cache, &c) == RF_OK && check_query(c, query, &u) == RF_OK ? rf_cache_attn_ws_bytes(c, u) : 0;
}

rf_status rf_cache_attn_fwd(const rf_cache* cache, const rf_cache_query* query, const void* q, const int32_t* q_len, const rf_schedule* sched,
                            void* o, float* lse, void* ws, size_t ws_bytes, int32_t* dev_status, void* cuda_stream) {
  return rf_cache_attn_fwd_origin(cache, query, q, q_len, nullptr, sched, o, lse, ws, ws_bytes, dev_status, cuda_stream);
}

rf_status rf_cache_attn_fwd_origin(const rf_cache* cache, const rf_cache_query* query, const void* q, const int32_t* q_len,
                                   const int32_t* block_origin, const rf_schedule* sched, void* o, float* lse, void* ws, size_t ws_bytes,
                                   int32_t* dev_status, void* cuda_stream) {
  RfCacheAttn a = {};
  rf_status st = check_cache(cache, &a.c);
  if (st == RF_OK) st = check_query(a.c, query, &a.u);
  if (st != RF_OK) return st;
  if (!aligned(q, 16) || !aligned(o, 16) || (lse != nullptr && !aligned(lse, 4))) return RF_ERR_INVALID_ARG;
  if (sched != nullptr) {
    if (sched->count == nullptr || sched->kv_tile == nullptr || sched->nQ != a.u.n_q || sched->nKmax < 1) return RF_ERR_INVALID_ARG;
    a.count = sched->count;
    a.pages = sched->kv_tile;
    a.n_k = sched->nKmax;
  }
  st = check_ws(ws, ws_bytes, rf_cache_attn_ws_bytes(a.c, a.u));
  if (st != RF_OK) return st;
  a.u.q = static_cast<const __nv_bfloat16*>(q);
  a.u.q_len = q_len;
  a.u.origin = block_origin;
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse;
  a.scale_log2 = (query->scale != 0.f ? query->scale : 1.f / sqrtf((float)a.c.D)) * 1.4426950408889634f;
  a.ws = static_cast<float*>(ws);
  a.dev_status = dev_status;
  return rf_launch_cache_attn(a, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
