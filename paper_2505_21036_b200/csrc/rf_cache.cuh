// The paged 8-bit K/V cache: what its kernels share.
#pragma once

#include <cuda_fp8.h>

#include "rf_common.cuh"

constexpr int kPage = RF_CACHE_PAGE;          // tokens of a page = query rows of a tile = the attention kernels' key tile
constexpr int kCacheMaxSeqs = 1024;           // a thread of the planning CTA each
constexpr int kCacheMaxPages = 1 << 19;       // two bitmaps of the pool in shared memory
constexpr int kSelectMaxPages = 1 << 14;      // a sequence's scores in shared memory

// The cache as the kernels see it (by value).
struct RfCache {
  int B, H, D, n_pages, max_pages;
  uint8_t *k, *v;
  float *k_scale, *v_scale, *k_sum;
  int32_t *table, *len;
};

// The queries of a call.
struct RfQueries {
  int M, G, rows, n_q;          // rows of q per query head, query heads per K/V head, G * M, tiles of kPage rows
  int causal;                   // tokens of a causal block, 0: none
  const __nv_bfloat16* q;       // [B, H, G * M, D]
  const int32_t* q_len;         // null: M
  const int32_t* origin;        // where the causal blocks begin, null: 0
};

__host__ __device__ __forceinline__ int rf_pages(int tokens) { return (tokens + kPage - 1) / kPage; }
// The page of a sequence that the x-th CTA of an append's grid writes to; -1: none.  (In pages: positions past a grid for 2^30 tokens pass 2^31.)
__host__ __device__ __forceinline__ int rf_append_page(int len, int add, unsigned x) {
  const int page = len / kPage + (int)x;
  return add > 0 && page < rf_pages(len + add) ? page : -1;
}

// A sequence's length as read, made safe.
__device__ __forceinline__ int rf_seq_len(const RfCache& c, int b, int32_t* dev_status) {
  const int n = c.len[b];
  if (n >= 0 && (long long)n <= (long long)c.max_pages * kPage) return n;
  rf_report(dev_status, RF_ERR_INVALID_ARG);
  return n < 0 ? 0 : c.max_pages * kPage;
}
__device__ __forceinline__ int rf_query_len(const RfQueries& u, int b, int32_t* dev_status) {
  if (u.q_len == nullptr) return u.M;
  const int n = u.q_len[b];
  if (n >= 0 && n <= u.M) return n;
  rf_report(dev_status, RF_ERR_INVALID_ARG);
  return n < 0 ? 0 : u.M;
}
__device__ __forceinline__ int rf_origin(const RfQueries& u, int b) { return u.origin == nullptr ? 0 : u.origin[b]; }
// Keys that query row i of a head sees.  Blocks of `causal` positions begin at `origin`, which may be any number; what lies before it is a block too.
__host__ __device__ __forceinline__ int rf_row_sees(int causal, int origin, int len, int q_len, int i) {
  if (causal == 0) return len;
  const int p = len - q_len + i;
  if (p < 0) return 0;
  const long long end = p < origin ? origin : (long long)origin + ((long long)(((unsigned)p - (unsigned)origin) / (unsigned)causal) + 1) * causal;
  return (int)(end < len ? end : (long long)len);
}
// (Out of line: two divisions, and its callers' code is to stay short.)  The most keys that any of the rows [r0, r0 + n) of a K/V head sees (they grow with a row's place in its head); -1 if
// all of them are padding.  Row r is row r % M of its query head.
static __host__ __device__ __noinline__ int rf_rows_see(const RfQueries& u, int origin, int len, int q_len, int r0, int n) {
  int i0 = r0, last;                               // the last place in a head among the rows that are there
  if (u.G != 1) i0 = r0 % u.M;
  const int end = i0 + (n < u.rows - r0 ? n : u.rows - r0);
  if (end <= u.M) last = i0 < q_len ? (end < q_len ? end : q_len) - 1 : -1;
  else last = i0 < q_len || end >= u.M + q_len ? q_len - 1 : end - u.M - 1;
  return last < 0 ? -1 : rf_row_sees(u.causal, origin, len, q_len, last);
}

// Physical page of a sequence's page c, made safe.
__device__ __forceinline__ int rf_page(const RfCache& a, int b, int c, int32_t* dev_status) {
  const int p = a.table[(size_t)b * a.max_pages + c];
  if (p >= 0 && p < a.n_pages) return p;
  rf_report(dev_status, RF_ERR_INVALID_ARG);
  return 0;
}

// Host side.
cudaError_t rf_launch_cache_append(const RfCache& c, const __nv_bfloat16* k, const __nv_bfloat16* v, int M, const int32_t* new_len,
                                   int32_t* ws, int32_t* dev_status, cudaStream_t st);
cudaError_t rf_launch_cache_fork(const RfCache& c, const int32_t* parent, int32_t* dev_status, cudaStream_t st);
cudaError_t rf_launch_cache_drop(const RfCache& c, const int32_t* first, const int32_t* count, const int32_t* max_len,
                                 int32_t* dev_status, cudaStream_t st);
cudaError_t rf_launch_cache_compact(const RfCache& c, int32_t* n_live, int32_t* ws, int32_t* dev_status, cudaStream_t st);
cudaError_t rf_launch_cache_select(const RfCache& c, const RfQueries& u, int keep_first, int keep_last, int top_k, int32_t* count,
                                   int32_t* pages, int n_k, int32_t* dev_status, cudaStream_t st);
size_t rf_cache_ws_words(const RfCache& c);

struct RfCacheAttn {
  RfCache c;
  RfQueries u;
  const int32_t *count, *pages;   // null: every page
  int n_k;                        // entries of a row of `pages`
  __nv_bfloat16* o;
  float* lse;                     // null: not wanted
  float scale_log2;
  float* ws;
  int32_t* dev_status;
};
// Tensor map over the pages' codes, [n_pages * H] blocks of 128 rows of D bytes; box = one block, rows swizzled by 128 bytes (64 at
// D = 64; at D = 96 a row takes 128 bytes in shared memory, the last 32 of them zeros).
bool rf_encode_pages_map(CUtensorMap* m, const uint8_t* codes, const RfCache& c);
size_t rf_cache_attn_ws_bytes(const RfCache& c, const RfQueries& u);
size_t rf_cache_chunk_ws_bytes(const RfCache& c, const RfQueries& u);
rf_status rf_launch_cache_chunk(const RfCacheAttn& a, cudaStream_t st);
rf_status rf_launch_cache_attn(const RfCacheAttn& a, cudaStream_t st);
