// Attention over the paged 8-bit cache for few query rows (single tokens; the rows of all query heads that share a K/V head).
//
// o = softmax(scale q k^T) v, over the keys that each row sees.  Every K and V byte is used by at most 16 rows, so the floor is
// the cache's bytes at the HBM rate: an SM has 1400 cycles for the 32 KB of a tile of 128 keys at D = 128.
// A producer warp streams the tiles into rings in shared memory by TMA (page by page, swizzled, 128 KB under way).  Eight warps
// take 16 keys of a tile each, on mma.sync with the keys as its 16 rows and the queries as its 8 columns (tcgen05 would spend 128 rows on
// them): S^T = K q^T, then O^T += V^T P^T with P^T turned round by movmatrix.  Codes are widened to fp16 in registers, exactly, by one
// conversion a pair (to bf16 it takes seven integer instructions and two products for four, and the integer pipe was what bound it: 152 us
// for 33 frames of 3600 tokens, 24 heads; 129 so, 5.7 TB/s).  So the other operands are fp16 too: a query row scaled by a power of two to a largest
// magnitude in [2^14, 2^15) (exact down to 2^-29 of that, 2^-40 of it beyond), and the weights times 2^15, whose largest is exact here
// (11 bits, to 2^-39 of the largest).  The scales of rows and pages are applied in fp32.  The order
// of a contraction is free, so the words are used as they lie: a word of K is four of the 16 terms of one instruction, and V's bytes
// of two keys are brought together by one byte permutation.  Up to 8 rows, two groups of eight warps take the tiles in turn, four warps
// to a scheduler (one group, and queries as rows of the product: 190 us for 33 frames of 3600 tokens, 24 heads, where the bytes take 112);
// 9 to 16 rows have two column blocks, which share the widened words, and one group, for its registers.
// Each warp keeps its own maxima and sums (fp32); they meet once per item.
#include <algorithm>

#include "rf_cache_attn.cuh"

using namespace sm100;
using namespace rf_cache_attn;

namespace {

enum { kFirst = 1, kLast = 2, kNothing = 4, kHeadPiece = 8, kTailPiece = 16, kEnd = 32 };

// An item and the key tiles that it walks; -1: all of its rows are padding.
struct TokenItem { CacheItem it; int tiles; };
template <int kRows>
static __device__ __noinline__ TokenItem token_item(const RfCacheAttn& a, int item) {
  TokenItem t;
  t.it = cache_item<kRows>(a, item);
  const int sees = rf_rows_see(a.u, t.it.origin, t.it.len, t.it.q_len, t.it.r0, kRows);
  t.tiles = sees < 0 ? -1 : a.count == nullptr ? rf_pages(sees) : listed(a, t.it, t.it.r0 / kPage);
  return t;
}
template <int D, int NB>
struct Cfg {
  static constexpr int ROWS = 8 * NB, GROUPS = NB == 1 ? 2 : 1, WARPS = 8 * GROUPS, THREADS = 32 * (WARPS + 1);
  static constexpr int PITCH = D == 64 ? 64 : 128;                  // bytes of a row in shared memory
  static constexpr uint32_t TILE = kPage * PITCH;
  static constexpr int SLOTS = D == 64 ? 8 : 4, STAGES = SLOTS / GROUPS;   // slots in all; of a group's ring
  static constexpr uint32_t JOIN = SLOTS * 2 * TILE;                // [WARPS][ROWS][D] float
  static constexpr uint32_t SUMS = JOIN + WARPS * ROWS * D * 4;     // [WARPS][ROWS] {m, l, l of the unrounded weights}
  static constexpr uint32_t BAR = SUMS + WARPS * ROWS * 16;
  static constexpr uint32_t REC = BAR + 8 * (2 * SLOTS + 2);
  static constexpr uint32_t MISC = REC + SLOTS * 32;                // (a Record each)
  static constexpr uint32_t TOTAL = MISC + 16 + sizeof(StretchScratch<TokenItem>);
  static constexpr uint32_t ALLOC = TOTAL + 1024;
  static_assert(ALLOC <= 227 * 1024, "shared memory of a CTA");
  static constexpr int PIECE = ROWS * (D + 4);                      // floats: O [ROWS][D], then {m, l, l exact, 0} per row
  // byte offset of 16-byte chunk c of row r
  static __device__ __forceinline__ uint32_t chunk(int r, int c) {
    return r * PITCH + ((D == 64 ? c ^ ((r >> 1) & 3) : c ^ (r & 7)) << 4);
  }
};

struct Record { int item, page, flags, len, q_len, origin; float ks, vs; };
static_assert(sizeof(Record) == 32, "Cfg::REC");

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
constexpr float kWeightUnit = 32768.f;           // the weights' largest

__device__ __forceinline__ uint32_t turn8x8(uint32_t x) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
  return d;
}

template <int kRows>
struct TokenPlaces {
  static constexpr int kRowsOf = kRows, kEnd = 6;     // what an item costs beside its tiles: Q, the meeting of the warps, its outputs
  using Info = TokenItem;
  static __device__ __forceinline__ TokenItem look(const RfCacheAttn& a, int item) { return token_item<kRows>(a, item); }
  static __device__ __forceinline__ int of(const TokenItem& t) { return t.tiles < 0 ? 0 : t.tiles + kEnd; }
};

struct Maps { CUtensorMap k, v; };

template <int D, int NB, bool LSE>
__global__ void __launch_bounds__((Cfg<D, NB>::THREADS), 1) rf_cache_token_kernel(const __grid_constant__ Maps maps, const __grid_constant__ RfCacheAttn a) {
  using C = Cfg<D, NB>;
  constexpr int kRows = C::ROWS, kWarps = C::WARPS;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  auto full = [&](int s) -> uint32_t { return base + C::BAR + 8u * s; };
  auto empty = [&](int s) -> uint32_t { return base + C::BAR + 8u * (C::SLOTS + s); };
  const uint32_t joined = base + C::BAR + 8u * (2 * C::SLOTS), read = joined + 8;   // all warps' rows of an item are in shared memory; they have been read
  volatile Record* records = reinterpret_cast<volatile Record*>(base_ptr + C::REC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + C::MISC);
  StretchScratch<TokenItem>* scratch = reinterpret_cast<StretchScratch<TokenItem>*>(base_ptr + C::MISC + 16);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
#pragma unroll 1
    for (int s = 0; s < C::SLOTS; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 8); }
    mbar_init(joined, kWarps);
    mbar_init(read, kWarps);
    *abort_flag = 0;
    mbar_init_fence();
  }
  if (tid == 32 * kWarps) { prefetch_tmap(&maps.k); prefetch_tmap(&maps.v); }
  rf_grid_wait();
  const Stretch st = stretch<TokenPlaces<kRows>, C::THREADS>(a, scratch);      // (its barriers also publish the mbarriers)
  const WaitCtx wc{abort_flag, a.dev_status};
  if (tid == 0) {
    int32_t* head = reinterpret_cast<int32_t*>(a.ws) + blockIdx.x * kHeadWords;
    head[0] = st.item;
    head[3] = st.cuts;
  }

  if (warp == kWarps) {
    // ------------------------------------------------------------ producer: tile t of a piece goes to group t mod GROUPS
    int sent[C::GROUPS] = {}, item = st.item;
    long long at = st.at;
    auto publish = [&](const Record& r, int group, bool bytes, int row) {   // lane 0
      const int n = sent[group], s = group * C::STAGES + n % C::STAGES;
      if (!wait_for(empty(s), ((n / C::STAGES) & 1) ^ 1, wc)) return;        // (the first round finds them free) abandoned: nothing more is fetched
      volatile Record* d = records + s;
      d->item = r.item; d->page = r.page; d->flags = r.flags; d->len = r.len; d->q_len = r.q_len; d->origin = r.origin;
      d->ks = r.ks; d->vs = r.vs;
      if (bytes) {
        const uint32_t to = base + s * 2 * C::TILE;
        mbar_expect_tx(full(s), 2 * C::TILE);
        tma_load_3d(to, &maps.k, 0, 0, row, full(s));
        tma_load_3d(to + C::TILE, &maps.v, 0, 0, row, full(s));
      } else {
        mbar_arrive(full(s));
      }
    };
#pragma unroll 1
    for (long long pos = st.lo; pos < st.hi; ++item) {
      const TokenItem ti = item == st.item ? scratch->info : token_item<kRows>(a, item);
      const CacheItem it = ti.it;
      const int tiles = ti.tiles;
      if (tiles < 0) continue;
      const int n = max(tiles, 1), begin = (int)(pos - at), end = (int)min((long long)n, st.hi - at);
      at += tiles + TokenPlaces<kRows>::kEnd;
      pos = min(at, st.hi);
      if (begin >= n) continue;                          // only the places of the item's end
      const int cut = (begin > 0 ? kHeadPiece : 0) | (end < n && begin == 0 ? kTailPiece : 0);
      const int32_t* list = a.count != nullptr ? a.pages + ((size_t)it.bh * a.u.n_q + it.r0 / kPage) * a.n_k : nullptr;
      const int pages = rf_pages(it.len);
      const int stop = max(end, begin + C::GROUPS);      // every group gets a record, with nothing in it if there is no tile
#pragma unroll 1
      for (int t0 = begin; t0 < stop; t0 += 32) {
        // a batch of tiles' entries, pages and scales: a lane each
        Record r;
        const int t = t0 + lane;
        int row = 0;
        r.item = item;
        r.page = t;
        r.flags = cut | (t < begin + C::GROUPS ? kFirst : 0) | (t >= stop - C::GROUPS ? kLast : 0);
        r.ks = r.vs = 0.f;
        if (t < end && t < tiles) {
          if (list != nullptr) r.page = list[t];
          if (r.page < 0 || r.page >= pages) {
            rf_report(a.dev_status, RF_ERR_INVALID_ARG);
            r.flags |= kNothing;
          } else {
            row = rf_page(a.c, it.b, r.page, a.dev_status) * a.c.H + it.bh % a.c.H;
            r.ks = a.c.k_scale[row];
            r.vs = a.c.v_scale[row];
          }
        } else {
          r.flags |= kNothing;
        }
        const int batch = min(32, stop - t0);
#pragma unroll 1
        for (int i = 0; i < batch; ++i) {
          Record s;
          s.item = item; s.len = it.len; s.q_len = it.q_len; s.origin = it.origin;
          s.page = __shfl_sync(0xffffffffu, r.page, i);
          s.flags = __shfl_sync(0xffffffffu, r.flags, i);
          s.ks = __shfl_sync(0xffffffffu, r.ks, i);
          s.vs = __shfl_sync(0xffffffffu, r.vs, i);
          const int row_i = __shfl_sync(0xffffffffu, row, i), group = (t0 + i - begin) % C::GROUPS;
          if (lane == 0) publish(s, group, !(s.flags & kNothing), row_i);
          __syncwarp();
          if (group == 0) ++sent[0]; else ++sent[C::GROUPS - 1];
        }
      }
    }
    if (lane == 0)
#pragma unroll 1
      for (int g = 0; g < C::GROUPS; ++g) publish(Record{0, 0, kEnd, 0, 0, 0, 0.f, 0.f}, g, false, 0);
  } else {
    // ------------------------------------------------------------ consumers: 16 keys of every tile of their group each
    const int g = lane >> 2, t = lane & 3, group = warp >> 3, slice = 16 * (warp & 7);
    uint32_t q[NB][D / 16][2];                 // B operands: row g of a block, four columns of every 16
    float o[NB][D / 16][4], m[NB][2], l[NB][2], lx[NB][2];   // of rows 2t, 2t + 1 of a block
    int sees[NB][2];
    float rs[NB][2];                           // those rows' factor of the scores
    uint32_t item_no = 0;
    CacheItem it = {};
    int stage = 0;
    uint32_t phase = 0;
#pragma unroll 1
    for (;;) {
      const int slot = group * C::STAGES + stage;
      // (the warp as a whole: after an abandoned wait its lanes may differ in what they saw)
      if (!__all_sync(0xffffffffu, wait_for(full(slot), phase, wc))) break;
      Record rec;
      {
        volatile const Record* r = records + slot;
        rec.item = r->item; rec.page = r->page; rec.flags = r->flags; rec.len = r->len; rec.q_len = r->q_len; rec.origin = r->origin;
        rec.ks = r->ks; rec.vs = r->vs;
      }
      if (rec.flags & kEnd) break;
      if (rec.flags & kFirst) {
        it.bh = rec.item;                                          // (all rows of a K/V head are one item here)
        it.r0 = 0;
        it.len = rec.len;
        it.q_len = rec.q_len;
        it.origin = rec.origin;
        const __nv_bfloat16* src = a.u.q + (size_t)it.bh * a.u.rows * D;
        int row_sees = -1;                                         // keys that row `lane` sees; -1: it is not there
        if (lane < kRows && it.r0 + lane < a.u.rows) {
          const int place = (it.r0 + lane) % a.u.M;
          if (place < it.q_len) row_sees = rf_row_sees(a.u.causal, it.origin, it.len, it.q_len, place);
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int r = it.r0 + 8 * nb + g;
          const bool there = __shfl_sync(0xffffffffu, row_sees, 8 * nb + g) >= 0;
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            uint2 x = make_uint2(0u, 0u);
            if (there) x = *reinterpret_cast<const uint2*>(src + (size_t)r * D + 16 * ks + 4 * t);
            q[nb][ks][0] = x.x;                                    // columns 0 and 1 of the four, as widen_low gives the keys'
            q[nb][ks][1] = x.y;
          }
          uint32_t most = 0u;                                      // the row's largest magnitude, as bf16 bits
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int i = 0; i < 2; ++i) most = max(most, max(q[nb][ks][i] & 0x7fffu, (q[nb][ks][i] >> 16) & 0x7fffu));
          most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
          most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
          const int e = most == 0u ? 0 : min(14 - ((int)(most >> 7) - 127), 126);
          const float up = __uint_as_float((uint32_t)(e + 127) << 23), down = a.scale_log2 * __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              q[nb][ks][i] = pack_f16(__uint_as_float(q[nb][ks][i] << 16) * up, __uint_as_float(q[nb][ks][i] & 0xffff0000u) * up);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            sees[nb][i] = max(__shfl_sync(0xffffffffu, row_sees, 8 * nb + 2 * t + i), 0);
            rs[nb][i] = __shfl_sync(0xffffffffu, down, 4 * (2 * t + i));
            m[nb][i] = -INFINITY;
            l[nb][i] = lx[nb][i] = 0.f;
          }
#pragma unroll
          for (int n = 0; n < D / 16; ++n) o[nb][n][0] = o[nb][n][1] = o[nb][n][2] = o[nb][n][3] = 0.f;
        }
      }
      if (!(rec.flags & kNothing)) {
        const uint32_t kt = base + slot * 2 * C::TILE, vt = kt + C::TILE;
        float s[NB][4] = {};                                       // keys g (0, 1) and g + 8 (2, 3) of the slice, rows 2t, 2t + 1
        {
          const int row = slice + (lane & 7) + ((lane >> 4) << 3), c0 = (lane >> 3) & 1;
#pragma unroll
          for (int ks = 0; ks < D / 16; ks += 2) {
            uint32_t x[4];
            ldmatrix4(kt + C::chunk(row, ks + c0), x);              // keys 0-7: chunks ks, ks + 1; keys 8-15 likewise
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t a0 = widen_low(x[i]), a1 = widen_low(x[2 + i]), a2 = widen_high(x[i]), a3 = widen_high(x[2 + i]);
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) mma16816(s[nb], a0, a1, a2, a3, q[nb][ks + i][0], q[nb][ks + i][1]);
            }
          }
        }
        // scores to weights
        const int key0 = rec.page * kPage + slice + g;
        uint32_t p[NB][2];                                         // P^T as the second product's B operand
        bool moved = false;
        float alpha[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float& x0 = s[nb][i];
            float& x1 = s[nb][2 + i];
            x0 = key0 < sees[nb][i] ? x0 * (rs[nb][i] * rec.ks) : -INFINITY;
            x1 = key0 + 8 < sees[nb][i] ? x1 * (rs[nb][i] * rec.ks) : -INFINITY;
            float mx = fmaxf(x0, x1);
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
            const float m_new = fmaxf(m[nb][i], mx), use = m_new == -INFINITY ? 0.f : m_new;
            alpha[nb][i] = m_new == m[nb][i] ? 1.f : ex2(m[nb][i] - use);      // 0 from -inf on
            moved |= m_new != m[nb][i];
            m[nb][i] = m_new;
            x0 = ex2(x0 - use + 15.f);                             // in units of 2^-15
            x1 = ex2(x1 - use + 15.f);
            if (LSE) lx[nb][i] = lx[nb][i] * alpha[nb][i] + (x0 + x1) * (1.f / kWeightUnit);
          }
          const uint32_t p0 = pack_f16(s[nb][0], s[nb][1]), p1 = pack_f16(s[nb][2], s[nb][3]);   // P V multiplies the rounded weights: they normalise O
          const float2 w0 = __half22float2(*reinterpret_cast<const __half2*>(&p0)), w1 = __half22float2(*reinterpret_cast<const __half2*>(&p1));
          l[nb][0] = l[nb][0] * alpha[nb][0] + (w0.x + w1.x) * (1.f / kWeightUnit);
          l[nb][1] = l[nb][1] * alpha[nb][1] + (w0.y + w1.y) * (1.f / kWeightUnit);
          p[nb][0] = turn8x8(p0);
          p[nb][1] = turn8x8(p1);
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int n = 0; n < D / 16; ++n) { o[nb][n][0] *= alpha[nb][0]; o[nb][n][1] *= alpha[nb][1]; o[nb][n][2] *= alpha[nb][0]; o[nb][n][3] *= alpha[nb][1]; }
        }
        const float vs = rec.vs * (1.f / kWeightUnit);
        const int valid = it.len - rec.page * kPage - slice;       // of this warp's keys; what lies behind them may be no numbers
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
          // word g + 8 j of keys 2t, 2t+1, 2t+8, 2t+9: columns 4 (g + 8 j) .. + 3, as rows g and g + 8 of two 16-row operands
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = lds32(vt + C::chunk(slice + 2 * t + (i & 1) + 8 * (i >> 1), 2 * j + (g >> 2)) + (g & 3) * 4);
          if (valid < 16) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (2 * t + (i & 1) + 8 * (i >> 1) >= valid) w[i] = 0u;
          }
#pragma unroll
          for (int hlf = 0; hlf < 2; ++hlf) {
            const uint32_t y = __byte_perm(w[0], w[1], hlf ? 0x7362 : 0x5140), z = __byte_perm(w[2], w[3], hlf ? 0x7362 : 0x5140);
            const uint32_t a0 = widen_low(y), a1 = widen_high(y), a2 = widen_low(z), a3 = widen_high(z);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              float tile[4] = {};
              mma16816(tile, a0, a1, a2, a3, p[nb][0], p[nb][1]);
#pragma unroll
              for (int i = 0; i < 4; ++i) o[nb][2 * j + hlf][i] += tile[i] * vs;
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(slot));
      if (++stage == C::STAGES) { stage = 0; phase ^= 1u; }
      if (!(rec.flags & kLast)) continue;

      // ---------------------------------------------------------- the item's (or piece's) end: the warps' rows meet
      const int n_rows = min(kRows, a.u.rows - it.r0);
      float* buf = reinterpret_cast<float*>(base_ptr + C::JOIN);
      float4* sums = reinterpret_cast<float4*>(base_ptr + C::SUMS);
      if (item_no > 0) wait_for(read, (item_no - 1) & 1, wc);    // the item before has been read
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) {
            l[nb][i] += __shfl_xor_sync(0xffffffffu, l[nb][i], d);
            if (LSE) lx[nb][i] += __shfl_xor_sync(0xffffffffu, lx[nb][i], d);
          }
          const int r = 8 * nb + 2 * t + i;
          if (r >= n_rows) continue;
          if (g == 0) sums[warp * kRows + r] = make_float4(m[nb][i], l[nb][i], lx[nb][i], 0.f);
          float* row = buf + ((size_t)warp * kRows + r) * D;
#pragma unroll
          for (int j = 0; j < D / 32; ++j)
            *reinterpret_cast<float4*>(row + 4 * (g + 8 * j)) =
                make_float4(o[nb][2 * j][i], o[nb][2 * j][2 + i], o[nb][2 * j + 1][i], o[nb][2 * j + 1][2 + i]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(joined);
      wait_for(joined, item_no & 1, wc);
      ++item_no;
      const bool piece = rec.flags & (kHeadPiece | kTailPiece);
      float* out = a.ws + head_floats(gridDim.x) + ((size_t)2 * blockIdx.x + (rec.flags & kTailPiece ? 1 : 0)) * C::PIECE;
#pragma unroll 1
      for (int i = tid; i < n_rows * (D / 4); i += 32 * kWarps) {
        const int r = i / (D / 4), d4 = i % (D / 4), place = (it.r0 + r) % a.u.M;
        float mm = -INFINITY, ll = 0.f, llx = 0.f;
#pragma unroll 4
        for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, sums[w * kRows + r].x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        const float use = mm == -INFINITY ? 0.f : mm;
#pragma unroll 4
        for (int w = 0; w < kWarps; ++w) {
          const float4 sm = sums[w * kRows + r], x = *reinterpret_cast<const float4*>(buf + ((size_t)w * kRows + r) * D + d4 * 4);
          const float f = ex2(sm.x - use);
          ll += sm.y * f; llx += sm.z * f;
          acc.x += x.x * f; acc.y += x.y * f; acc.z += x.z * f; acc.w += x.w * f;
        }
        if (piece) {
          __stcg(reinterpret_cast<float4*>(out + (size_t)r * D) + d4, acc);
          if (d4 == 0) __stcg(reinterpret_cast<float4*>(out + (size_t)kRows * D) + r, make_float4(mm, ll, llx, 0.f));
        } else if (place < it.q_len) {
          const float inv = ll == 0.f ? 0.f : 1.f / ll;            // (a sum that is no number stays one)
          const size_t at_row = (size_t)it.bh * a.u.rows + it.r0 + r;
          if (!rf_in_bounds(at_row, (unsigned long long)a.c.B * a.c.H * a.u.rows, a.dev_status)) continue;
          *reinterpret_cast<uint2*>(a.o + at_row * D + d4 * 4) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
          if (LSE && d4 == 0) a.lse[at_row] = (mm + log2f(llx)) * 0.6931471805599453f;
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(read);
    }
  }
  __syncthreads();
  if (tid == 0 && *abort_flag) __nanosleep(20000);   // let abandoned copies land before shared memory is released
}

// Joins the pieces of the items that the stretches cut.  CTA x looks at the cut between stretches x and x + 1 and works if it is the
// first one inside its item; blockIdx.y is the row.
template <int D, int NB, bool LSE>
__global__ void __launch_bounds__(D) rf_cache_join_kernel(const __grid_constant__ RfCacheAttn a, int ctas) {
  constexpr int kRows = 8 * NB, PIECE = Cfg<D, NB>::PIECE;
  __shared__ float red[2][D / 32];
  __shared__ int last;
  extern __shared__ float weight[];              // [ctas]
  rf_grid_wait();
  const int x = blockIdx.x + 1, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = blockIdx.y;
  const int32_t* heads = reinterpret_cast<const int32_t*>(a.ws);
  const int32_t* mine = heads + x * kHeadWords;
  if (!mine[3]) return;
  // the item begins in the stretch before, unless that one begins inside it too
  const int32_t* prev = mine - kHeadWords;
  if (prev[3] && prev[0] == mine[0]) return;
  const int n = cuts_from(heads, x, ctas, &last);
  const CacheItem it = cache_item<kRows>(a, mine[0]);
  const int row = it.r0 + r;
  if (row >= a.u.rows || row % a.u.M >= it.q_len) return;
  const float* pieces = a.ws + head_floats(ctas);
  // piece 0 is the one that stretch x - 1 ends in, piece i > 0 the one that stretch x + i - 1 begins in
  auto at = [&](int i) -> const float* { return pieces + (i == 0 ? (size_t)2 * (x - 1) + 1 : (size_t)2 * (x + i - 1)) * PIECE; };
  float mm = -INFINITY;
#pragma unroll 1
  for (int i = tid; i <= n; i += D) {
    const float m = __ldcg(at(i) + (size_t)kRows * D + r * 4);
    weight[i] = m;
    mm = fmaxf(mm, m);
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, d));
  if (lane == 0) red[0][warp] = mm;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < D / 32; ++i) mm = fmaxf(mm, red[0][i]);
  const float use = mm == -INFINITY ? 0.f : mm;
  float l = 0.f, lx = 0.f, acc = 0.f;
#pragma unroll 4
  for (int i = 0; i <= n; ++i) {
    const float4 sm = __ldcg(reinterpret_cast<const float4*>(at(i) + (size_t)kRows * D) + r);
    const float f = ex2(weight[i] - use);
    l += sm.y * f;
    lx += sm.z * f;
    acc += __ldcg(at(i) + (size_t)r * D + tid) * f;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const size_t at_row = (size_t)it.bh * a.u.rows + row;
  if (!rf_in_bounds(at_row, (unsigned long long)a.c.B * a.c.H * a.u.rows, a.dev_status)) return;
  a.o[at_row * D + tid] = __float2bfloat16_rn(acc * inv);
  if (LSE && tid == 0) a.lse[at_row] = (mm + log2f(lx)) * 0.6931471805599453f;
}

constexpr int kMostRows = 16;
int blocks_of(const RfQueries& u) { return u.rows <= 8 ? 1 : 2; }

// One CTA an SM; fewer where there is nothing to share out (a bound on the places of the line from the sizes alone).
int token_ctas(const RfCache& c) { return (int)std::min<long long>((long long)c.B * c.H * (c.max_pages + 2ll), 148); }

template <int D, int NB, bool LSE>
rf_status launch(const RfCacheAttn& a, cudaStream_t st) {
  using C = Cfg<D, NB>;
  static bool configured[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return RF_ERR_CUDA;
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    if (cudaFuncSetAttribute(rf_cache_token_kernel<D, NB, LSE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::ALLOC) != cudaSuccess)
      return RF_ERR_CUDA;
    configured[dev] = true;
  }
  Maps maps;
  if (!rf_encode_pages_map(&maps.k, a.c.k, a.c) || !rf_encode_pages_map(&maps.v, a.c.v, a.c)) return RF_ERR_CUDA;
  const int ctas = token_ctas(a.c);
  if (rf_launch(rf_cache_token_kernel<D, NB, LSE>, dim3(ctas), C::THREADS, C::ALLOC, st, maps, a) != cudaSuccess) return RF_ERR_CUDA;
  if (ctas == 1) return RF_OK;
  return rf_launch(rf_cache_join_kernel<D, NB, LSE>, dim3(ctas - 1, a.u.rows), D, sizeof(float) * (ctas + 1), st, a, ctas) == cudaSuccess ? RF_OK : RF_ERR_CUDA;
}
template <int D>
rf_status launch(const RfCacheAttn& a, cudaStream_t st) {
  if (blocks_of(a.u) == 1) return a.lse != nullptr ? launch<D, 1, true>(a, st) : launch<D, 1, false>(a, st);
  return a.lse != nullptr ? launch<D, 2, true>(a, st) : launch<D, 2, false>(a, st);
}

}  // namespace

namespace {
// Whether a call's query rows are few: see the top of this file and of rf_cache_chunk.cu.
bool few_rows(const RfQueries& u) { return u.rows <= kMostRows; }
}  // namespace

size_t rf_cache_attn_ws_bytes(const RfCache& c, const RfQueries& u) {
  if (!few_rows(u)) return rf_cache_chunk_ws_bytes(c, u);
  const int ctas = token_ctas(c);
  return (head_floats(ctas) + (size_t)2 * ctas * 8 * blocks_of(u) * (c.D + 4)) * sizeof(float);
}

rf_status rf_launch_cache_attn(const RfCacheAttn& a, cudaStream_t st) {
  if (!few_rows(a.u)) return rf_launch_cache_chunk(a, st);
  switch (a.c.D) {
    case 64: return launch<64>(a, st);
    case 96: return launch<96>(a, st);
    case 128: return launch<128>(a, st);
  }
  return RF_ERR_UNSUPPORTED;
}
