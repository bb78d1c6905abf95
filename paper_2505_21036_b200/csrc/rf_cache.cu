// The paged 8-bit K/V cache: appending, page operations, selection of pages.
//
// All of its state is on the device and every call is a fixed sequence of launches, so whole steps can be captured.  Which
// pages are free follows from the page table alone (those that no row names), so there are no reference counts that could
// disagree with it: a planning kernel of one CTA marks the named pages in a bitmap in shared memory, where a second
// bitmap tells the pages that are named more than once.
#include <math.h>

#include "rf_cache.cuh"

namespace {

constexpr int kPlanThreads = 1024;

// Exclusive prefix sum over the CTA's kPlanThreads values; `total` for everybody.  s: 33 ints of shared memory.
__device__ __forceinline__ int block_scan(int v, int* s, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();                       // the last scan's sums have been read
  if (lane == 31) s[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int t = s[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, t, d);
      if (lane >= d) t += y;
    }
    s[lane] = t;
  }
  __syncthreads();
  total = s[31];
  return x - v + (warp ? s[warp - 1] : 0);
}

// Workspace words: per sequence {old length, new tokens, page that held its partly filled last page}, a few counts, then
// two lists of n_pages words.
enum { kWsCount = 0, kWsHead = 64 };
struct PlanWs {
  int32_t *count, *old_len, *n_new, *src, *list, *to;
};
__host__ __device__ __forceinline__ PlanWs plan_ws(int32_t* ws, int B, int n_pages) {
  PlanWs w;
  w.count = ws + kWsCount;
  w.old_len = ws + kWsHead;
  w.n_new = w.old_len + B;
  w.src = w.n_new + B;
  w.list = w.src + B;
  w.to = w.list + n_pages;
  return w;
}

// Marks the pages that the table names; `lens` in shared memory, all in range; *most_pages (shared memory too) becomes the
// longest row's number of pages.  False for everybody if an entry is none.
__device__ __forceinline__ bool mark_pages(const RfCache& c, const int* lens, uint32_t* used, uint32_t* twice, int words, int* most_pages) {
#pragma unroll 1
  for (int i = threadIdx.x; i < words; i += kPlanThreads) {
    used[i] = 0u;
    if (twice != nullptr) twice[i] = 0u;
  }
  if (threadIdx.x == 0) *most_pages = 0;
  __syncthreads();
  if (threadIdx.x < c.B) atomicMax(most_pages, rf_pages(lens[threadIdx.x]));
  __syncthreads();
  bool bad = false;
  const int most = *most_pages;
  // Over the rows' used columns only.  (The products fit: n_seqs * max_pages < 2^33, in 64 bits.)
  const long long n = (long long)c.B * most;
#pragma unroll 1
  for (long long i = threadIdx.x; i < n; i += kPlanThreads) {
    const int b = (int)(i / most), col = (int)(i - (long long)b * most);
    if (col >= rf_pages(lens[b])) continue;
    const int p = c.table[(size_t)b * c.max_pages + col];
    if (p < 0 || p >= c.n_pages) {
      bad = true;
      continue;
    }
    const uint32_t bit = 1u << (p & 31), before = atomicOr(&used[p >> 5], bit);
    if (twice != nullptr && (before & bit)) atomicOr(&twice[p >> 5], bit);
  }
  return !__syncthreads_or(bad);
}

// ------------------------------------------------------------------------------------------------ append
// Pages for the tokens that come, and the sequences' new lengths.  One CTA: what it does is a chain of a dozen round trips
// to the L2, about 5 us, whatever the pool's size up to some ten thousand pages.
constexpr int kFew = 1024;
__global__ void __launch_bounds__(kPlanThreads) rf_cache_plan_kernel(RfCache c, int M, const int32_t* new_len, int32_t* ws, int32_t* dev_status) {
  extern __shared__ uint32_t bits[];
  __shared__ int scan[33], lens[kCacheMaxSeqs], need_at[kCacheMaxSeqs + 1], most, few[kFew];
  const int tid = threadIdx.x, words = (c.n_pages + 31) / 32;
  uint32_t *used = bits, *twice = bits + words;
  const PlanWs w = plan_ws(ws, c.B, c.n_pages);
  rf_grid_trigger();
  rf_grid_wait();

  int len = 0, add = 0;
  bool bad = false, full = false;
  if (tid < c.B) {
    len = c.len[tid];
    add = new_len != nullptr ? new_len[tid] : M;
    const long long most = (long long)c.max_pages * kPage;
    bad = len < 0 || len > most || add < 0 || add > M;
    full = !bad && (long long)len + add > min(most, 0x7fffffffll);
    lens[tid] = bad ? 0 : len;
  }
  // the sequence's partly filled last page (looked at once the table is known to be in order)
  int old_page = -1;
  if (tid < c.B && !bad && !full && add > 0 && len % kPage != 0) old_page = c.table[(size_t)tid * c.max_pages + len / kPage];
  bad = __syncthreads_or(bad);
  if (!bad) bad = !mark_pages(c, lens, used, twice, words, &most);
  // fresh pages of this thread's sequence; its partly filled last page is among them if others name it too
  int need = 0, first_new = 0, shared_page = 0;
  if (!bad && tid < c.B && add > 0 && !full) {
    first_new = rf_pages(len);
    need = rf_pages(len + add) - first_new;
    if (len % kPage != 0) {
      shared_page = (twice[old_page >> 5] >> (old_page & 31)) & 1u;
      need += shared_page;
    }
  }
  int total, n_free, at = block_scan(need, scan, total);
  const int per = (words + kPlanThreads - 1) / kPlanThreads, w0 = min(tid * per, words), w1 = min(w0 + per, words);
  auto free_of = [&](int i) -> uint32_t {
    const uint32_t f = ~used[i];
    return i == words - 1 && (c.n_pages & 31) ? f & ((1u << (c.n_pages & 31)) - 1u) : f;
  };
  int mine = 0;
#pragma unroll 1
  for (int i = w0; i < w1; ++i) mine += __popc(free_of(i));
  int rank = block_scan(mine, scan, n_free);
  full = __syncthreads_or(full) || total > n_free;
  if (bad || full) {
    if (tid == 0) rf_report(dev_status, bad ? RF_ERR_INVALID_ARG : RF_ERR_CACHE_FULL);
    if (tid < c.B) w.n_new[tid] = 0;
    return;
  }
  int32_t* list = total <= kFew ? few : w.list;              // fresh pages in the order they are handed out
  if (tid < c.B) need_at[tid] = at;
  if (tid == 0) need_at[c.B] = total;
#pragma unroll 1
  for (int i = w0; i < w1 && rank < total; ++i)
#pragma unroll 1
    for (uint32_t f = free_of(i); f != 0u && rank < total; f &= f - 1u) list[rank++] = i * 32 + __ffs(f) - 1;
  if (tid < c.B) {
    w.old_len[tid] = len;
    w.n_new[tid] = add;
    w.src[tid] = old_page;
    c.len[tid] = len + add;
    lens[tid] = first_new - shared_page;       // the first column that gets a fresh page
  }
  __syncthreads();
#pragma unroll 1
  for (int i = tid; i < total; i += kPlanThreads) {
    int lo = 0, hi = c.B - 1;                   // the last sequence whose pages begin at i or before
#pragma unroll 1
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (need_at[mid] <= i) lo = mid; else hi = mid - 1;
    }
    const int col = lens[lo] + i - need_at[lo];
    if (rf_in_bounds(col, c.max_pages, dev_status)) c.table[(size_t)lo * c.max_pages + col] = list[i];
  }
}

// e4m3 code -> its value in units of 2^-9 (an integer of at most 18 bits and a sign).
__device__ __forceinline__ int code_units(uint32_t code) {
  const int e = (code >> 3) & 15, m = code & 7;
  const int v = e == 0 ? m : (8 + m) << (e - 1);
  return code & 0x80 ? -v : v;
}
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 <= e <= 127

// Eight codes of a row.
__device__ __forceinline__ uint2 encode8(const float (&f)[8]) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __nv_cvt_float2_to_fp8x2(make_float2(f[2 * i], f[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
}
__device__ __forceinline__ void decode8(uint2 code, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)((i < 2 ? code.x : code.y) >> (16 * (i & 1))), __NV_E4M3)));
    f[2 * i] = x.x;
    f[2 * i + 1] = x.y;
  }
}

// One page of one head, K or V.  A thread takes 8 columns (16 bytes in, 8 out) of every 16th row, all loads first; the new tokens'
// largest magnitude has to be known before the first code, so they are held in registers and read once.  Bound by HBM for
// whole frames (6 bytes a pair of values of K and V); for single tokens by the two launches.  The page's old tokens, in a sequence's first
// page, are gone through in a loop of their own: written again only where they move to another page or another scale, K's read for the sum.
// The sum of the codes does not depend on how the page was filled: a thread's eight rows are exact in fp32 (multiples of 2^-9 below 2^12),
// and the threads' sums are added as integers.
template <int D>
__global__ void __launch_bounds__(2 * D) rf_cache_write_kernel(RfCache c, const __nv_bfloat16* kx, const __nv_bfloat16* vx, int M, const int32_t* ws,
                                                               int32_t* dev_status) {
  constexpr int kCols = D / 8, kPasses = kPage / 16, kThreads = 2 * D;
  static_assert(kCols * 16 == kThreads, "a pass is 16 rows");
  __shared__ int red[kThreads / 32], sums[D];
  const int tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z >> 1, col = tid % kCols, row0 = tid / kCols;
  const bool keys = (blockIdx.z & 1) == 0;
  const PlanWs w = plan_ws(const_cast<int32_t*>(ws), c.B, c.n_pages);
  rf_grid_trigger();
  rf_grid_wait();
  const int add = w.n_new[b], len = w.old_len[b], page = rf_append_page(len, add, blockIdx.x);
  if (page < 0) return;
  const int t0 = page * kPage;
  const int held = max(0, min(kPage, len - t0)), end = min(kPage, len + add - t0);
  const int dst = c.table[(size_t)b * c.max_pages + page];
  if (!rf_in_bounds(dst, c.n_pages, dev_status)) return;
  const int src = held ? w.src[b] : dst;
  if (tid < D) sums[tid] = 0;

  const __nv_bfloat16* x = (keys ? kx : vx) + (((size_t)b * c.H + h) * M + (t0 - len)) * D + col * 8;
  const size_t block = (size_t)kPage * D;
  uint8_t* data = keys ? c.k : c.v;
  uint8_t* out = data + ((size_t)dst * c.H + h) * block + col * 8;
  float* scales = keys ? c.k_scale : c.v_scale;
  const int e_old = held ? min(max((int)(__float_as_uint(scales[(size_t)src * c.H + h]) >> 23) - 127, -100), 100) : -100;
  uint4 v[kPasses];
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int r = row0 + 16 * p;
    v[p] = r >= held && r < end ? *reinterpret_cast<const uint4*>(x + (size_t)r * D) : make_uint4(0u, 0u, 0u, 0u);
  }
  // largest finite magnitude of the new tokens, as bf16 bits
  uint32_t most = 0u;
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const uint32_t* u = &v[p].x;
#pragma unroll
    for (int i = 0; i < 4; ++i) most = __vmaxu2(most, u[i] & 0x7fff7fffu);
  }
  most = max(most >> 16, most & 0xffffu);
  if (most >= 0x7f80u) {                                     // something is not finite: NaN becomes zero, infinities saturate
    rf_report(dev_status, RF_ERR_NOT_FINITE);
    most = 0u;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      uint32_t* u = &v[p].x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((u[i] & 0x7fffu) > 0x7f80u) u[i] &= 0xffff0000u;
        if (((u[i] >> 16) & 0x7fffu) > 0x7f80u) u[i] &= 0xffffu;
        const uint32_t lo = u[i] & 0x7fffu, hi = (u[i] >> 16) & 0x7fffu;
        most = max(most, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
      }
    }
  }
  most = __reduce_max_sync(0xffffffffu, most);
  if ((tid & 31) == 0) red[tid >> 5] = (int)most;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) most = max(most, (uint32_t)red[i]);
  // 448 = 1.75 * 2^8, so with m * 2^E the largest magnitude e is E - 8, or E - 7 where m > 1.75; subnormal ones end at -100
  const int e = min(max(max((int)(most >> 7) - 127 - ((most & 127u) > 96u ? 7 : 8), e_old), -100), 100);
  const float inv = pow2f(-e);
  float acc[8] = {};
#pragma unroll
  for (int p = 0; p < kPasses; ++p) {
    const int r = row0 + 16 * p;
    if (r < held || r >= end) continue;
    float f[8];
    const uint32_t* u = &v[p].x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16) * inv;
      f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u) * inv;
    }
    const uint2 code = encode8(f);
    *reinterpret_cast<uint2*>(out + (size_t)r * D) = code;
    if (keys) {
      decode8(code, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += f[i];
    }
  }
  const bool moves = src != dst || e > e_old;                // old tokens get another place or scale
  if (held && (keys || moves)) {
    const uint8_t* old = data + ((size_t)src * c.H + h) * block + col * 8;
    const float again = pow2f(max(e_old - e, -126));
#pragma unroll 4
    for (int r = row0; r < held; r += 16) {
      uint2 code = *reinterpret_cast<const uint2*>(old + (size_t)r * D);
      float f[8];
      decode8(code, f);
      if (e > e_old) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= again;
        code = encode8(f);
        decode8(code, f);
      }
      if (moves) *reinterpret_cast<uint2*>(out + (size_t)r * D) = code;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += f[i];
    }
  }
  const size_t side = (size_t)dst * c.H + h;
  if (tid == 0) scales[side] = pow2f(e);
  if (!keys) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) atomicAdd(&sums[col * 8 + i], __float2int_rn(acc[i] * 512.f));
  __syncthreads();
  if (tid < D) c.k_sum[side * D + tid] = (float)sums[tid] * 0.001953125f * pow2f(e);
}

// ------------------------------------------------------------------------------------------------ fork, drop
__device__ __forceinline__ bool broken_len(const RfCache& c, int len) { return len < 0 || (long long)len > (long long)c.max_pages * kPage; }

// Thirty-two columns of the table: the old rows are taken into shared memory and written back in their new places.
__global__ void __launch_bounds__(256) rf_cache_fork_kernel(RfCache c, const int32_t* parent, int32_t* dev_status) {
  extern __shared__ int rows[];                       // [B][32], then the lengths in CTA 0
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, col = blockIdx.x * 32 + lane;
  rf_grid_trigger();
  rf_grid_wait();
  bool bad = false;
#pragma unroll 1
  for (int b = tid; b < c.B; b += 256) bad |= parent[b] < -1 || parent[b] >= c.B || broken_len(c, c.len[b]);
#pragma unroll 1
  for (int b = warp; b < c.B; b += 8)
    if (col < c.max_pages) rows[b * 32 + lane] = c.table[(size_t)b * c.max_pages + col];
  int* lens = rows + c.B * 32;
  if (blockIdx.x == 0)
#pragma unroll 1
    for (int b = tid; b < c.B; b += 256) lens[b] = c.len[b];
  if (__syncthreads_or(bad)) {
    if (blockIdx.x == 0 && tid == 0) rf_report(dev_status, RF_ERR_INVALID_ARG);
    return;
  }
#pragma unroll 1
  for (int b = warp; b < c.B; b += 8) {
    const int p = parent[b];
    if (p >= 0 && p != b && col < c.max_pages) c.table[(size_t)b * c.max_pages + col] = rows[p * 32 + lane];
  }
  if (blockIdx.x == 0)
#pragma unroll 1
    for (int b = tid; b < c.B; b += 256) c.len[b] = parent[b] < 0 ? 0 : lens[parent[b]];
}

__global__ void __launch_bounds__(256) rf_cache_drop_kernel(RfCache c, const int32_t* first, const int32_t* count, const int32_t* max_len, int32_t* dev_status) {
  const int tid = threadIdx.x, b = blockIdx.x;
  rf_grid_trigger();
  rf_grid_wait();
  bool bad = false;
#pragma unroll 1
  for (int i = tid; i < c.B; i += 256) {
    if (max_len != nullptr) bad |= max_len[i] < 0;
    if (first != nullptr) bad |= first[i] < 0 || count[i] < 0;
    bad |= broken_len(c, c.len[i]);                    // (a length that another CTA has written already is in order before and after)
  }
  int len = c.len[b];                                  // (read by everybody before the barrier, written after it)
  if (__syncthreads_or(bad)) {
    if (b == 0 && tid == 0) rf_report(dev_status, RF_ERR_INVALID_ARG);
    return;
  }
  if (max_len != nullptr) len = min(len, max_len[b]);
  const int pages = rf_pages(len);
  if (first != nullptr) {
    const int from = min(first[b], pages), n = min(count[b], pages - from);
    if (n > 0) {
      int32_t* row = c.table + (size_t)b * c.max_pages;
#pragma unroll 1
      for (int base = from + n; base < pages; base += 256) {      // ascending: a stretch is read before it is written over
        const int i = base + tid, p = i < pages ? row[i] : 0;
        __syncthreads();
        if (i < pages) row[i - n] = p;
        __syncthreads();
      }
      len -= min(len, (from + n) * kPage) - from * kPage;
    }
  }
  if (tid == 0) c.len[b] = len;
}

// ------------------------------------------------------------------------------------------------ compact
__global__ void __launch_bounds__(kPlanThreads) rf_cache_compact_plan_kernel(RfCache c, int32_t* n_live, int32_t* ws, int32_t* dev_status) {
  extern __shared__ uint32_t bits[];
  __shared__ int scan[33], lens[kCacheMaxSeqs], most;
  const int tid = threadIdx.x, words = (c.n_pages + 31) / 32;
  uint32_t* used = bits;
  const PlanWs w = plan_ws(ws, c.B, c.n_pages);
  rf_grid_trigger();
  rf_grid_wait();
  bool bad = false;
  if (tid < c.B) {
    const int len = c.len[tid];
    bad = len < 0 || (long long)len > (long long)c.max_pages * kPage;
    lens[tid] = bad ? 0 : len;
  }
  bad = __syncthreads_or(bad);
  if (!bad) bad = !mark_pages(c, lens, used, nullptr, words, &most);
  if (bad) {
    if (tid == 0) {
      rf_report(dev_status, RF_ERR_INVALID_ARG);
      *w.count = 0;
      *n_live = -1;
    }
    return;
  }
  const int per = (words + kPlanThreads - 1) / kPlanThreads, w0 = min(tid * per, words), w1 = min(w0 + per, words);
  int mine = 0, live, moves, n;
#pragma unroll 1
  for (int i = w0; i < w1; ++i) mine += __popc(used[i]);
  block_scan(mine, scan, live);
  // bits of word i that lie before page `live`
  auto below = [&](int i) -> uint32_t {
    const int d = live - i * 32;
    return d >= 32 ? 0xffffffffu : d <= 0 ? 0u : (1u << d) - 1u;
  };
  int holes = 0, movers = 0;
#pragma unroll 1
  for (int i = w0; i < w1; ++i) {
    holes += __popc(~used[i] & below(i));
    movers += __popc(used[i] & ~below(i));
  }
  int hole_at = block_scan(holes, scan, n), mover_at = block_scan(movers, scan, moves);   // n == moves
#pragma unroll 1
  for (int i = w0; i < w1; ++i)
#pragma unroll 1
    for (uint32_t f = ~used[i] & below(i); f != 0u; f &= f - 1u) w.to[hole_at++] = i * 32 + __ffs(f) - 1;
#pragma unroll 1
  for (int i = w0; i < w1; ++i)
#pragma unroll 1
    for (uint32_t f = used[i] & ~below(i); f != 0u; f &= f - 1u) w.list[mover_at++] = i * 32 + __ffs(f) - 1;
  if (tid == 0) {
    *w.count = moves;
    *n_live = live;
  }
  __syncthreads();
  const long long all = (long long)c.B * most;
#pragma unroll 1
  for (long long i = tid; i < all; i += kPlanThreads) {
    const int b = (int)(i / most), col = (int)(i - (long long)b * most);
    if (col >= rf_pages(lens[b])) continue;
    int32_t* entry = c.table + (size_t)b * c.max_pages + col;
    const int p = *entry;
    if (p < live) continue;
    int lo = 0, hi = moves - 1;                 // its place among the moving pages, which ascend
#pragma unroll 1
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (w.list[mid] < p) lo = mid + 1; else hi = mid;
    }
    *entry = w.to[lo];
  }
}

// Copies page list[i] to page to[i]: a work item is one head of one moving page, K or V, 16 KB at D = 128.  Sources lie
// behind the live pages' number and destinations before it, so no item reads what another writes.
__global__ void __launch_bounds__(256) rf_cache_move_kernel(RfCache c, const int32_t* ws, int32_t* dev_status) {
  rf_grid_trigger();
  rf_grid_wait();
  const PlanWs w = plan_ws(const_cast<int32_t*>(ws), c.B, c.n_pages);
  const int moves = *w.count, tid = threadIdx.x, n16 = kPage * c.D / 16;
  const long long items = (long long)moves * c.H * 2;
#pragma unroll 1
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int m = (int)(it / (2 * c.H)), r = (int)(it % (2 * c.H)), h = r >> 1;
    const bool keys = (r & 1) == 0;
    const int from = w.list[m], to = w.to[m];
    if (!rf_in_bounds(from, c.n_pages, dev_status) || !rf_in_bounds(to, c.n_pages, dev_status)) continue;
    const size_t sf = (size_t)from * c.H + h, st = (size_t)to * c.H + h;
    uint8_t* data = keys ? c.k : c.v;
    const uint4* s = reinterpret_cast<const uint4*>(data + sf * kPage * c.D);
    uint4* d = reinterpret_cast<uint4*>(data + st * kPage * c.D);
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (tid + i * 256 < n16) v[i] = s[tid + i * 256];
    float sum = 0.f;
    if (keys && tid < c.D) sum = c.k_sum[sf * c.D + tid];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (tid + i * 256 < n16) d[tid + i * 256] = v[i];
    if (keys && tid < c.D) c.k_sum[st * c.D + tid] = sum;
    if (tid == 0) {
      float* scales = keys ? c.k_scale : c.v_scale;
      scales[st] = scales[sf];
    }
  }
}

// ------------------------------------------------------------------------------------------------ select
// A CTA takes up to 8 tiles of query rows of a K/V head: their sums, their products with every page's key sum, the top_k best of each,
// the lists in order.  Scores are in 64 bits: a page's place must not hang on the order of a summation, and two scores that differ in
// exact arithmetic hardly ever agree to 1e-16.  What bounds it: widening the key sums to 64 bits (16 a cycle and SM) and the 64-bit
// products, so the tiles are the columns and the pages the rows of a 64-bit matrix product: a lane widens a number once for eight tiles and
// holds its part of the tiles' sums in registers.  (29 tiles x 931 pages x 24 heads: 136 us with a tile a CTA, 67 with a lane a page and
// four tiles a CTA, whose loads touched 32 rows at a time, 40 so.  A single tile, which would waste seven of the eight columns, is multiplied
// without matrix products: a token each of 32 heads 21 and 16 us.)
constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;

__device__ __forceinline__ uint64_t ordered(double x) {   // monotone; NaN below everything
  if (isnan(x)) return 0ull;
  const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
  return u >> 63 ? ~u : u | (1ull << 63);
}

// D (8 pages x 8 tiles) += A (8 x 4) B (4 x 8): a lane holds A[lane / 4][lane % 4], B[lane % 4][lane / 4], D[lane / 4][2 (lane % 4) + 0, 1].
__device__ __forceinline__ void mma_f64(double (&d)[2], double a, double b) {
  asm volatile("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};" : "+d"(d[0]), "+d"(d[1]) : "d"(a), "d"(b));
}

template <int D, int T>
__global__ void __launch_bounds__(kSelThreads, 1) rf_cache_select_kernel(RfCache c, RfQueries u, int keep_first, int keep_last, int top_k, int32_t* count,
                                                                      int32_t* pages, int n_k, int32_t* dev_status) {
  constexpr int kOf = kSelWarps / T, kTeam = 32 * kOf;     // warps and threads that work on a tile
  extern __shared__ uint64_t keys[];                       // [T][pages of the sequence]
  __shared__ double part[kSelWarps][D];
  __shared__ double pooled[T][D];
  __shared__ __align__(16) float tail_sum[D];
  __shared__ int hist[T][256], state[T][4], warp_n[kSelWarps][2], cand[T + 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int mine = warp / kOf, rank = tid % kTeam, wrank = warp % kOf;     // this thread's tile, and its place in the tile's team
  const int tile = blockIdx.x * T + mine, h = blockIdx.y, b = blockIdx.z;
  rf_grid_wait();
  const int len = rf_seq_len(c, b, dev_status), q_len = rf_query_len(u, b, dev_status);
  const int sees = tile < u.n_q ? rf_rows_see(u, rf_origin(u, b), len, q_len, tile * kPage, kPage) : -1;
  const size_t row = ((size_t)b * c.H + h) * u.n_q + min(tile, u.n_q - 1);
  const int n = min(rf_pages(max(sees, 0)), kSelectMaxPages);             // pages in which some row of the tile sees a key
  const int first_end = min(keep_first, n), last_begin = max(n - min(keep_last, n), first_end);
  const int rest = last_begin - first_end, best = min(top_k, rest);
  const bool scored = best > 0 && best < rest;
  if (rank == 0) cand[mine] = scored ? last_begin : 0;
  if (tid == 0) cand[T] = 0;
  __syncthreads();
  if (rank == 0 && scored) atomicMax(&cand[T], last_begin);
  __syncthreads();
  const int most = cand[T];                                 // pages to be scored: [keep_first, most)
  uint64_t threshold = ~0ull;
  int equal_allowed = 0;                                    // pages of exactly the threshold's score that are taken, lowest first
  if (most > 0) {                                           // (the same for the whole CTA)
    {
      // the sums of the tile's rows: a lane's columns (two, four, or at D = 96 every 32nd), a warp every kOf-th row, eight of them under way
      constexpr int kMine = D / 32, kAhead = 8;
      auto column = [&](int i) { return D == 96 ? lane + 32 * i : lane * kMine + i; };
      double acc[kMine] = {};
      const __nv_bfloat16* q = u.q + (((size_t)b * c.H + h) * u.rows + (size_t)tile * kPage) * D;
      const int rows = scored ? min(kPage, u.rows - tile * kPage) : 0;
#pragma unroll 1
      for (int r0 = wrank; r0 < rows; r0 += kOf * kAhead) {
        uint16_t v[kAhead][kMine];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int r = r0 + k * kOf, at = tile * kPage + r;
          const bool there = r < rows && (u.G == 1 ? at : at % u.M) < q_len;
          const __nv_bfloat16* x = q + (size_t)(there ? r : 0) * D;
          if (D == 128) {
            const uint2 t = there ? *reinterpret_cast<const uint2*>(x + lane * 4) : make_uint2(0u, 0u);
            v[k][0] = (uint16_t)t.x; v[k][1] = (uint16_t)(t.x >> 16); v[k][kMine - 2] = (uint16_t)t.y; v[k][kMine - 1] = (uint16_t)(t.y >> 16);
          } else if (D == 64) {
            const uint32_t t = there ? *reinterpret_cast<const uint32_t*>(x + lane * 2) : 0u;
            v[k][0] = (uint16_t)t; v[k][1] = (uint16_t)(t >> 16);
          } else {
#pragma unroll
            for (int i = 0; i < kMine; ++i) v[k][i] = there ? *reinterpret_cast<const uint16_t*>(x + column(i)) : (uint16_t)0;
          }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
          for (int i = 0; i < kMine; ++i) acc[i] += (double)__uint_as_float((uint32_t)v[k][i] << 16);
      }
#pragma unroll
      for (int i = 0; i < kMine; ++i) part[warp][column(i)] = acc[i];
    }
    // A last page that is not full is summed up from its codes: it may be part of a page that another sequence has filled
    // further, or that was fuller when it was written.
    const int tail = len % kPage != 0 && most == rf_pages(len) ? most - 1 : -1;
    if (tail >= 0 && tid < D) {
      const size_t side = (size_t)rf_page(c, b, tail, dev_status) * c.H + h;
      const uint8_t* codes = c.k + side * kPage * D + tid;
      int sum = 0;
#pragma unroll 8
      for (int r = 0; r < len % kPage; ++r) sum += code_units(codes[r * D]);
      tail_sum[tid] = (float)sum * 0.001953125f * c.k_scale[side];
    }
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < T * D; i += kSelThreads) {
      const int t = i / D, d = i % D;
      double x = 0.0;
#pragma unroll
      for (int k = 0; k < kOf; ++k) x += part[t * kOf + k][d];
      pooled[t][d] = x;
    }
    __syncthreads();
    // four columns of every 16 for a lane, so that it reads 16 bytes at a time: a sum's order is free
    const int g = lane >> 2, q4 = lane & 3;
    double w[D / 16][4];
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
      for (int k = 0; k < 4; ++k) w[d][k] = T == 1 || g < T ? pooled[T == 1 ? 0 : g % T][16 * d + 4 * q4 + k] : 0.0;
#pragma unroll 1
    for (int c0 = keep_first + warp * 8; c0 < most; c0 += kSelWarps * 8) {
      const int col = c0 + g;
      const bool there = col < most;
      const float4* x = reinterpret_cast<const float4*>(col == tail ? tail_sum : c.k_sum + ((size_t)(there ? rf_page(c, b, col, dev_status) : 0) * c.H + h) * D) + q4;
      float4 v[D / 16];
#pragma unroll
      for (int d = 0; d < D / 16; ++d) v[d] = there ? x[4 * d] : make_float4(0.f, 0.f, 0.f, 0.f);
      double dot[2] = {};
      if constexpr (T == 1) {                               // one column: as multiplications, the four lanes of a page add theirs up
        double sum[4] = {};
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          sum[0] += (double)v[d].x * w[d][0];
          sum[1] += (double)v[d].y * w[d][1];
          sum[2] += (double)v[d].z * w[d][2];
          sum[3] += (double)v[d].w * w[d][3];
        }
        dot[0] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        dot[0] += __shfl_xor_sync(0xffffffffu, dot[0], 1);
        dot[0] += __shfl_xor_sync(0xffffffffu, dot[0], 2);
      } else {
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          mma_f64(dot, (double)v[d].x, w[d][0]);
          mma_f64(dot, (double)v[d].y, w[d][1]);
          mma_f64(dot, (double)v[d].z, w[d][2]);
          mma_f64(dot, (double)v[d].w, w[d][3]);
        }
      }
      const double tokens = (double)min(kPage, len - col * kPage);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (2 * q4 + i < T && there && col < cand[2 * q4 + i < T ? 2 * q4 + i : 0]) keys[(size_t)(2 * q4 + i) * c.max_pages + col] = ordered(dot[i] / tokens);
    }
    __syncthreads();
  }
  // From here on every tile's team works by itself.
  auto team_sync = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(1 + mine), "n"(kTeam) : "memory"); };
  const uint64_t* key = keys + (size_t)mine * c.max_pages;
  if (scored) {
    // the best-th largest: eight bits at a time
    uint64_t prefix = 0ull;
    int need = best;
#pragma unroll 1
    for (int shift = 56; shift >= 0; shift -= 8) {
#pragma unroll 1
      for (int i = rank; i < 256; i += kTeam) hist[mine][i] = 0;
      team_sync();
#pragma unroll 1
      for (int base = first_end + wrank * 32; base < last_begin; base += kTeam) {
        const int i = base + lane;
        const uint64_t k = i < last_begin ? key[i] : 0ull;
        const bool in = i < last_begin && (shift == 56 || (k >> (shift + 8)) == prefix);
        const int bin = in ? (int)(k >> shift) & 255 : -1;
        int same;                                           // the leading digits are alike: one addition for the warp
        __match_all_sync(0xffffffffu, bin, &same);
        if (same) {
          if (in && lane == 0) atomicAdd(&hist[mine][bin], 32);
        } else if (in) {
          atomicAdd(&hist[mine][bin], 1);
        }
      }
      team_sync();
      if (wrank == 0) {                                     // from the top bin down: where `need` is reached
        int v[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[i] = hist[mine][255 - (lane * 8 + i)];
          sum += v[i];
        }
        int before = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int y = __shfl_up_sync(0xffffffffu, before, d);
          if (lane >= d) before += y;
        }
        before -= sum;
        if (before < need && before + sum >= need) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (before < need && before + v[i] >= need) {
              state[mine][0] = 255 - (lane * 8 + i);
              state[mine][1] = need - before;
              state[mine][2] = v[i];
              break;
            }
            before += v[i];
          }
        }
      }
      team_sync();
      prefix = prefix << 8 | (uint64_t)state[mine][0];
      need = state[mine][1];
      const int in_bin = state[mine][2];
      threshold = prefix << shift;
      equal_allowed = need;
      if (in_bin == need) {                                 // the whole bin is taken: everything from its lower end on
        equal_allowed = 0x7fffffff;
        break;
      }
    }
  }
  // the list, in order
  int out = 0, ties = 0;
#pragma unroll 1
  for (int base = 0; base < n; base += kTeam) {
    const int col = base + rank;
    const bool always = col < n && (col < first_end || col >= last_begin);
    const bool candidate = col < n && !always && best > 0;
    const uint64_t k = candidate && scored ? key[col] : 0ull;
    // (where the whole last bin is taken `threshold` is its lower end and equal_allowed has no bound)
    const bool tie = candidate && scored && equal_allowed != 0x7fffffff && k == threshold;
    const uint32_t tie_mask = __ballot_sync(0xffffffffu, tie);
    if (lane == 0) warp_n[warp][0] = __popc(tie_mask);
    team_sync();
    int tie_rank = ties + __popc(tie_mask & ((1u << lane) - 1u)), tie_all = 0;
#pragma unroll
    for (int i = 0; i < kOf; ++i) {
      if (i < wrank) tie_rank += warp_n[mine * kOf + i][0];
      tie_all += warp_n[mine * kOf + i][0];
    }
    bool take = always;
    if (candidate) take = !scored ? true : tie ? tie_rank < equal_allowed : equal_allowed == 0x7fffffff ? k >= threshold : k > threshold;
    const uint32_t mask = __ballot_sync(0xffffffffu, take);
    if (lane == 0) warp_n[warp][1] = __popc(mask);
    team_sync();
    int at = out + __popc(mask & ((1u << lane) - 1u)), all = 0;
#pragma unroll
    for (int i = 0; i < kOf; ++i) {
      if (i < wrank) at += warp_n[mine * kOf + i][1];
      all += warp_n[mine * kOf + i][1];
    }
    if (take && at < n_k && rf_in_bounds(at, n_k, dev_status)) pages[row * n_k + at] = col;
    out += all;
    ties += tie_all;
    team_sync();
  }
  if (rank == 0 && tile < u.n_q) count[row] = min(out, n_k);
}

// On a kernel's first use on a device, whatever this call's size: the 48 KB that need no asking are of static and dynamic memory together.
template <typename K>
cudaError_t allow_smem(K kernel, bool (&done)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || (dev < 64 && done[dev])) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 192 * 1024);
  if (e == cudaSuccess && dev < 64) done[dev] = true;
  return e;
}

}  // namespace

size_t rf_cache_ws_words(const RfCache& c) { return kWsHead + 3 * (size_t)c.B + 2 * (size_t)c.n_pages; }

cudaError_t rf_launch_cache_append(const RfCache& c, const __nv_bfloat16* k, const __nv_bfloat16* v, int M, const int32_t* new_len,
                                   int32_t* ws, int32_t* dev_status, cudaStream_t st) {
  static bool done[64] = {};
  const size_t smem = 2 * sizeof(uint32_t) * rf_cdiv(c.n_pages, 32);
  cudaError_t e = allow_smem(rf_cache_plan_kernel, done);
  if (e != cudaSuccess) return e;
  e = rf_launch(rf_cache_plan_kernel, dim3(1), kPlanThreads, smem, st, c, M, new_len, ws, dev_status);
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)((M - 1 + kPage - 1) / kPage + 1), c.H, 2 * c.B);   // pages that M tokens from any place on can touch
  switch (c.D) {
    case 64: return rf_launch(rf_cache_write_kernel<64>, grid, 128, 0, st, c, k, v, M, ws, dev_status);
    case 96: return rf_launch(rf_cache_write_kernel<96>, grid, 192, 0, st, c, k, v, M, ws, dev_status);
    default: return rf_launch(rf_cache_write_kernel<128>, grid, 256, 0, st, c, k, v, M, ws, dev_status);
  }
}

cudaError_t rf_launch_cache_fork(const RfCache& c, const int32_t* parent, int32_t* dev_status, cudaStream_t st) {
  static bool done[64] = {};
  const size_t smem = (size_t)c.B * 33 * sizeof(int);
  cudaError_t e = allow_smem(rf_cache_fork_kernel, done);
  if (e != cudaSuccess) return e;
  return rf_launch(rf_cache_fork_kernel, dim3(rf_cdiv(c.max_pages, 32)), 256, smem, st, c, parent, dev_status);
}

cudaError_t rf_launch_cache_drop(const RfCache& c, const int32_t* first, const int32_t* count, const int32_t* max_len,
                                 int32_t* dev_status, cudaStream_t st) {
  return rf_launch(rf_cache_drop_kernel, dim3(c.B), 256, 0, st, c, first, count, max_len, dev_status);
}

cudaError_t rf_launch_cache_compact(const RfCache& c, int32_t* n_live, int32_t* ws, int32_t* dev_status, cudaStream_t st) {
  static bool done[64] = {};
  const size_t smem = sizeof(uint32_t) * rf_cdiv(c.n_pages, 32);
  cudaError_t e = allow_smem(rf_cache_compact_plan_kernel, done);
  if (e != cudaSuccess) return e;
  e = rf_launch(rf_cache_compact_plan_kernel, dim3(1), kPlanThreads, smem, st, c, n_live, ws, dev_status);
  if (e != cudaSuccess) return e;
  const long long most = (long long)c.n_pages * c.H;      // of n pages at most half move, two items a head
  return rf_launch(rf_cache_move_kernel, dim3((unsigned)(most < 148 * 8 ? most : 148 * 8)), 256, 0, st, c, ws, dev_status);
}

cudaError_t rf_launch_cache_select(const RfCache& c, const RfQueries& u, int keep_first, int keep_last, int top_k, int32_t* count,
                                   int32_t* pages, int n_k, int32_t* dev_status, cudaStream_t st) {
  // Eight tiles a CTA share the key sums; one where the scores of eight do not fit in shared memory or there is only one.
  const bool eight = u.n_q > 1 && 8 * sizeof(uint64_t) * (size_t)c.max_pages <= 128 * 1024;
  const size_t smem = (eight ? 8 : 1) * sizeof(uint64_t) * (size_t)c.max_pages;
  auto go = [&](auto kernel, bool (&done)[64]) -> cudaError_t {
    const cudaError_t e = allow_smem(kernel, done);
    if (e != cudaSuccess) return e;
    return rf_launch(kernel, dim3(rf_cdiv(u.n_q, eight ? 8 : 1), c.H, c.B), kSelThreads, smem, st, c, u, keep_first, keep_last, top_k, count, pages, n_k, dev_status);
  };
  static bool done[6][64] = {};
  switch (c.D) {
    case 64: return eight ? go(rf_cache_select_kernel<64, 8>, done[0]) : go(rf_cache_select_kernel<64, 1>, done[1]);
    case 96: return eight ? go(rf_cache_select_kernel<96, 8>, done[2]) : go(rf_cache_select_kernel<96, 1>, done[3]);
    default: return eight ? go(rf_cache_select_kernel<128, 8>, done[4]) : go(rf_cache_select_kernel<128, 1>, done[5]);
  }
}
