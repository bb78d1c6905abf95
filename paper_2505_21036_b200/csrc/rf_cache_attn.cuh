// What the attention kernels over the cache share: how the work is cut, how pieces are left and joined, how codes are widened.
//
// The work of a call is one line of key tiles: the items (a K/V head's block of query rows) one after another, each with the
// tiles that it lists.  The line is cut into as many equal stretches as there are CTAs, wherever that falls, so every SM gets
// the same number of tiles whatever the lengths are; an item that is cut leaves unnormalised pieces in the workspace, which
// a second kernel joins in order.  Lengths and lists are on the device, so every CTA sums the items up for itself.
#pragma once

#include "rf_cache.cuh"
#include "rf_sm100.cuh"

namespace rf_cache_attn {

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A bounded wait (see mbar_wait_long) whose slow part is called, not inlined.  A kernel here starts with cold instruction caches, as a
// layer runs other kernels in between, and fetches its code from the L2 line by line: what is not straight on the way is kept short or
// out of line.
static __device__ __noinline__ bool wait_slowly(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* dev_status, int tiles) {
  return sm100::mbar_wait_long(bar, parity, sm100::WaitCtx{abort_flag, dev_status}, tiles);
}
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, const sm100::WaitCtx& w, int tiles = 0) {
  return sm100::mbar_try(bar, parity) || wait_slowly(bar, parity, w.abort_flag, w.dev_status, tiles);
}

// An item: rows [r0, r0 + kRows) of K/V head bh.
struct CacheItem { int b, bh, r0, len, q_len, origin; };
template <int kRows>
__device__ __forceinline__ CacheItem cache_item(const RfCacheAttn& a, int item) {
  const int blocks = rf_cdiv(a.u.rows, kRows);
  CacheItem it;
  it.bh = item / blocks;
  it.r0 = (item - it.bh * blocks) * kRows;
  it.b = it.bh / a.c.H;
  it.len = rf_seq_len(a.c, it.b, a.dev_status);
  it.q_len = rf_query_len(a.u, it.b, a.dev_status);
  it.origin = rf_origin(a.u, it.b);
  return it;
}
// Entries of the list of a tile of query rows.
__device__ __forceinline__ int listed(const RfCacheAttn& a, const CacheItem& it, int tile) {
  return it.len == 0 ? 0 : min(max(a.count[(size_t)it.bh * a.u.n_q + tile], 0), a.n_k);
}
// A CTA's stretch [lo, hi) of the line, and the item that lo lies in (which begins at place `at`; behind the places of its tiles lie
// some that stand for what an item costs beside them, at least one, so that a row block that sees nothing has its outputs written).
// cuts: lo lies among that item's tiles, behind the first.
struct Stretch { long long lo, hi, at; int item, cuts; };
template <typename Info>
struct StretchScratch { long long sums[33]; Stretch st; Info info; };    // info: that item, looked up

// Called by all threads of the CTA (kThreads of them, whole warps).  Places::look(a, item): the item; Places::of(info): its places on the
// line, kEnd of them at its end for itself; 0 for an item whose rows are all padding.
template <typename Places, int kThreads>
__device__ __forceinline__ Stretch stretch(const RfCacheAttn& a, StretchScratch<typename Places::Info>* s) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int items = a.c.B * a.c.H * rf_cdiv(a.u.rows, Places::kRowsOf), per = rf_cdiv(items, kThreads);
  const int i0 = min(tid * per, items), i1 = min(i0 + per, items);
  long long mine = 0;
  typename Places::Info info = {};
#pragma unroll 1
  for (int i = i0; i < i1; ++i) {
    info = Places::look(a, i);
    mine += Places::of(info);
  }
  long long x = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) s->sums[warp] = x;
  __syncthreads();
  long long before = x - mine, total = 0;
#pragma unroll 1
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += s->sums[w];
    total += s->sums[w];
  }
  // no more stretches than places: the ones in use are the first, and none of them is empty
  const long long n = min((long long)gridDim.x, max(total, 1ll)), x0 = min((long long)blockIdx.x, n), x1 = min(x0 + 1, n);
  const long long lo = total * x0 / n, hi = total * x1 / n;
  if (tid == 0 && lo == hi) s->st = Stretch{lo, hi, lo, items, 0};
  if (lo < hi && before <= lo && lo < before + mine) {
    long long at = before;
    int i = i0;
#pragma unroll 1
    for (;; ++i) {
      if (per > 1) info = Places::look(a, i);              // (a thread's only item is at hand)
      const int p = Places::of(info);
      if (lo < at + p) {
        s->st = Stretch{lo, hi, at, i, at < lo && lo < at + p - Places::kEnd};
        s->info = info;
        break;
      }
      at += p;
    }
  }
  __syncthreads();
  return s->st;
}

// These kernels, and the selection, do not let the next kernel's CTAs in before they end (no rf_grid_trigger): such CTAs took places that the
// attention's own, one to an SM with most of its shared memory, then waited for (selection and attention of single tokens, 25 us each by
// themselves: 88 us together with the triggers, 50 without).

// Workspace: a head per CTA {the item its stretch begins in, -, -, whether it begins inside it}, then two
// pieces per CTA: that of the item its stretch begins inside, that of the item its stretch ends inside.
constexpr int kHeadWords = 4;
// Stretches x, x + 1, .. that begin inside the item that stretch x begins inside.  Called by all threads of the CTA; *s: shared memory.
__device__ __forceinline__ int cuts_from(const int32_t* heads, int x, int ctas, int* s) {
  if (threadIdx.x == 0) *s = ctas - x;
  __syncthreads();
  const int item = heads[x * kHeadWords];
#pragma unroll 1
  for (int i = x + 1 + threadIdx.x; i < ctas; i += blockDim.x)
    if (!heads[i * kHeadWords + 3] || heads[i * kHeadWords] != item) {
      atomicMin(s, i - x);
      break;
    }
  __syncthreads();
  return *s;
}
__host__ __device__ __forceinline__ size_t head_floats(int ctas) { return ((size_t)ctas * kHeadWords + 63) / 64 * 64; }

// Bytes 0 and 1, bytes 2 and 3 of a word of codes as fp16 pairs.
__device__ __forceinline__ uint32_t widen_low(uint32_t x) {
  uint32_t d;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(d) : "r"(x));
  return d;
}
__device__ __forceinline__ uint32_t widen_high(uint32_t x) {
  uint32_t d;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(d) : "r"(x));
  return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 t = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&t);
}
}  // namespace rf_cache_attn
