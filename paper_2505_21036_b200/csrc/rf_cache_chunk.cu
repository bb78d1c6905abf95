// Attention over the paged 8-bit cache for chunks of query rows, on tcgen05 / TMEM / TMA.
//
// o = softmax(scale q k^T) v over the keys that each row sees.  From some dozens of rows on the products bound it, not the
// cache's bytes.  An item is 256 query rows of one K/V head in two tiles of 128 (two "streams"), as in the attention
// kernel over whole clips, whose softmax it shares; what differs is where K and V come from: pages of e4m3 codes.
//
// Scores: K's codes go to the tensor cores as they are (kind::f8f6f4), and each query row, which is bf16, as a sum of two 8-bit
// numbers.  With the row scaled by a power of two to a largest magnitude in (224, 448], hi = e4m3(q) leaves at most 8 units of q's last place, which
// e5m2 holds exactly: q = hi + lo exactly from 2^-6 up (2^-14 of the row's largest), and below to within 2^-14 (2^-21.8 of the largest, the
// order of an fp32 sum's own rounding).  hi K^T + lo K^T costs what one bf16 product costs, K takes half the shared memory, and nothing has
// to be widened; the page's scale and the row's go into the softmax's factor.
// Values: V is widened to fp16 by four warps (one conversion a pair of codes, exact), once for the 256 rows, and laid out in shared memory in
// the swizzled form that tcgen05 reads, beside the softmax.  A page's scale has to go into V or into the weights, as O adds up over pages:
// V is held in units of 2^ref, ref the scale of the piece's first page, until a page's scale is more than 2^7 above it or 2^15 below, where fp16
// would not hold it exactly: that page's scale is the next ref, and O is rescaled, as for a new maximum, in the rows that take
// something of the page.  (Rare where a layer's pages are of like size.)  Only pages more than 2^60 below the largest unit so far lose places.
// The weights are fp16 too: 2^7 at the running maximum, at most 2^15, exact to 11 bits down to 2^-21 of the maximum and to 2^-31 of it in
// steps; a row of a million keys loses 2^-12 of its weight at most.
// (V to bf16 in seven integer instructions and two products for four codes: 2050 cycles of the widening warps' 3470 a tile, beside the softmax
// on the same integer pipes; 24 heads, 2040 rows, 32 896 keys, D = 128: 784 us, to fp16 764 (1070 TFLOP/s), with the widening left out 686.  K
// widened as well, by the same four warps: 1090.  Repeated for a second the board's power limits it: 870
// to 896, by box.  The units that follow the pages cost 0.5 % of that, and 2 % where rows are ragged and lse is wanted.)
// Warp roles:
//   warps 0-3, 4-7   softmax of streams 0 and 1 (one thread per query row)
//   warp 8           pages: walks the item's tiles, looks their pages and scales up (eight at a time), fetches Q and the codes by TMA
//   warp 9           issues the tcgen05.mma
//   warps 12-15      split an item's Q, widen V
// The last group's code is kept short, in rolled loops over shared memory: beside the softmax's two thousand instructions long stretches
// of straight code come in from the L2 line by line.  (Q split in unrolled code from global loads: 25 000 cycles an item, most of them
// waits for instructions.)
// The work is cut into equal stretches of tiles, one per SM (rf_cache_attn.cuh); cut items are joined by a second kernel.
#include <algorithm>

#include "rf_attn_softmax.cuh"
#include "rf_cache_attn.cuh"

namespace {

using namespace sm100;
using namespace rf_attn;
using rf_cache_attn::CacheItem;
using rf_cache_attn::Stretch;
using rf_cache_attn::StretchScratch;
using rf_cache_attn::head_floats;
using rf_cache_attn::kHeadWords;
using rf_cache_attn::pack_f16;
using rf_cache_attn::widen_high;
using rf_cache_attn::widen_low;

constexpr int kRows = 2 * BM, kThreads = 512;
constexpr int kPagesWarp = 8, kMmaWarp = 9, kWidenWarp = 12;
constexpr int kItemSlots = 2, kItemWords = 16, kItemReaders = 8;   // readers: the softmax warps
constexpr int kBatch = 8, kUnroll = 2;
constexpr uint32_t kMore = 4, kLast = 8, kFirst = 16;
enum { kHeadPiece = 1, kTailPiece = 2 };
// Register split: 2 x 128 softmax threads, 128 of the pages / MMA warpgroup, 128 that widen.  Checked like the clip kernel's
// (see rf_regs_ok): against the register file here, against what the launch really owns on the host.
constexpr int kRegsSoftmax = 200, kRegsControl = 48, kRegsWiden = 64;
static_assert(256 * kRegsSoftmax + 128 * kRegsControl + 128 * kRegsWiden <= 65536, "setmaxnreg split exceeds the register file of an SM");
#define RF_REGS_SOFTMAX() asm volatile("setmaxnreg.inc.sync.aligned.u32 200;")
#define RF_REGS_CONTROL() asm volatile("setmaxnreg.dec.sync.aligned.u32 48;")
#define RF_REGS_WIDEN() asm volatile("setmaxnreg.dec.sync.aligned.u32 64;")
static_assert(kRegsSoftmax == 200 && kRegsControl == 48 && kRegsWiden == 64, "keep the macros in step");

// Lazy raising of the running maximum as in the clip kernel, but within what fp16 weights hold: a weight at the maximum is 2^kTop, one that
// exceeds it by kRaise 2^15.
constexpr float kTop = 7.0f, kRaise = 8.0f, kRaiseMargin = 3.0f;
// V's reference scale, in log2: a page's scale is at most kMostUp above it (the largest code is then 57344) and at least -kLeastUp below it
// (the least code 2^-24), where V is exact in fp16.  It goes up and down with the pages, but not more than kMostDown below where it has been for the rows,
// whose O would not stay in fp32 otherwise: 2^30 keys of weight 2^15 and value 2^16 are below 2^61 of it.
constexpr int kMostUp = 7, kLeastUp = -15, kMostDown = 60;
constexpr float kNothing = 33.0f;                           // a score that far below the maximum has a weight of zero (2^kTop * 2^-32 is half of the least fp16 number):
                                                            // a row that takes nothing of a tile keeps its unit, and its bits
constexpr int kSpec = 32;

// What an item costs beside its tiles (Q, the first scores, the last product, its outputs or pieces), in tiles.
constexpr int kItemPlaces = 6;

// An item and the two streams' lists: how long they are.  there: some row is no padding.
struct ChunkItem { CacheItem it; int n0, n1; bool there; };
static __device__ __noinline__ ChunkItem chunk_item(const RfCacheAttn& a, int item) {
  ChunkItem c;
  c.it = rf_cache_attn::cache_item<kRows>(a, item);
  int n[2];
  c.there = false;
#pragma unroll 1
  for (int j = 0; j < 2; ++j) {
    const int r = c.it.r0 + j * BM, sees = r < a.u.rows ? rf_rows_see(a.u, c.it.origin, c.it.len, c.it.q_len, r, BM) : -1;
    c.there |= sees >= 0;
    const int tiles = sees < 0 ? 0 : a.count == nullptr ? rf_pages(sees) : rf_cache_attn::listed(a, c.it, r / kPage);
    if (j == 0) n[0] = tiles; else n[1] = tiles;
  }
  c.n0 = n[0];
  c.n1 = n[1];
  return c;
}
struct ChunkPlaces {
  static constexpr int kRowsOf = kRows, kEnd = kItemPlaces;
  using Info = ChunkItem;
  static __device__ __forceinline__ ChunkItem look(const RfCacheAttn& a, int item) { return chunk_item(a, item); }
  static __device__ __forceinline__ int of(const ChunkItem& c) { return c.there ? max(c.n0, c.n1) + kItemPlaces : 0; }
};

// TMEM columns and V's layout are those of the clip kernel (rf_attn.cu: Cfg), where they are explained: V in blocks of VBOX columns with a block of ones behind them whose product is
// the row sum of the rounded weights, P on top of S (D = 96 / 128) or in columns of its own (D = 64).
template <int D>
struct Cfg {
  // Q (its two parts) and K: 128 rows of PITCH bytes, swizzled by their pitch; at D = 96 the last 32 bytes are not used
  static constexpr int PITCH = D == 64 ? 64 : 128;
  static constexpr uint32_t TILE = 128 * PITCH;
  static __host__ __device__ constexpr uint32_t qchunk(int row, int c) { return row * PITCH + ((D == 64 ? c ^ ((row >> 1) & 3) : c ^ (row & 7)) << 4); }
  static constexpr bool S_EARLY = D == 64;
  static constexpr int NK = D == 128 ? 2 : 3, NV = D == 64 ? 3 : 2, NS = 2;    // slots of K, of V, of V's codes
  static constexpr int VBOX = D == 96 ? 32 : 64;
  static constexpr uint32_t VROW = VBOX * 2, VBLK = 128 * VROW, VLOAD = D / VBOX * VBLK, VTILE = VLOAD + VBLK;
  static constexpr int NPV = D + 16;
  static constexpr int PARTS = D == 64 ? 1 : 2;
  static __host__ __device__ constexpr int cut(int p) { return p * (BN / PARTS); }
  static __host__ __device__ constexpr uint32_t vchunk(int row, int c) { return row * VROW + ((VBOX == 64 ? c ^ (row & 7) : c ^ ((row >> 1) & 3)) << 4); }
  // Q: stream 0 hi, lo, stream 1 hi, lo; the rows come in as bf16 in the same place, 64 columns where hi goes and the others where lo goes,
  // or at D = 64 in a place of their own
  static constexpr uint32_t Q = 0, RAW = 4 * TILE, K0 = RAW + (D == 64 ? 2 * 128 * 128 : 0), VS0 = K0 + NK * TILE, V0 = VS0 + NS * TILE, BAR = V0 + NV * VTILE;
  static constexpr int B_Q = 0, B_QE = 1, B_QR = 2, B_KF = 3, B_KE = B_KF + NK, B_VF = B_KE + NK, B_VE = B_VF + NV, B_SF = B_VE + NV, B_PF = B_SF + 2,
                       B_OF = B_PF + 2 * PARTS, B_SE = B_OF + 2, B_IF = B_SE + 2, B_IE = B_IF + kItemSlots, B_CF = B_IE + kItemSlots,
                       B_CE = B_CF + NS, B_COUNT = B_CE + NS;
  static constexpr uint32_t MISC = BAR + 8 * B_COUNT;
  static constexpr uint32_t ITEM = (MISC + 16 + 15) / 16 * 16;
  static constexpr uint32_t RECORD = ITEM + kItemSlots * kItemWords * 4;    // what goes with a slot of V's codes: 4 words
  static constexpr uint32_t FLAGS = RECORD + NS * 16;                       // a tile's flags and V's reference for the MMA thread, by K slot
  static constexpr uint32_t REF = FLAGS + 16;                               // V's reference of a stream's tile
  static constexpr uint32_t WINDOW = REF + 16;                            // kBatch entries of the two lists, then a batch of the union
  static constexpr uint32_t ROWEXP = WINDOW + 4 * kBatch * 4;               // by item slot: exponent field of what undoes a row's scaling
  static_assert(ROWEXP % 8 == 0 && (ROWEXP + kItemSlots * kRows) % 8 == 0, "alignment");
  static constexpr uint32_t SCRATCH = ROWEXP + kItemSlots * kRows;
  static constexpr uint32_t TOTAL = SCRATCH + sizeof(StretchScratch<ChunkItem>);
  static constexpr uint32_t ALLOC = TOTAL + 1024;
  static_assert(ALLOC <= 227 * 1024, "shared memory of a CTA");
  static constexpr bool S_SHARED = D != 96;
  static constexpr uint32_t S_COL0 = 0, S_COL1 = S_SHARED ? 96 : 128, S_END = S_COL1 + 128, TMEM_COLS = 512;
  static constexpr uint32_t P_COL0 = S_EARLY ? S_END : S_COL0, P_COL1 = S_EARLY ? S_END + 64 : S_COL1 + 64;
  static constexpr uint32_t O_COL0 = S_EARLY ? S_END + 128 : S_END, O_COL1 = O_COL0 + NPV;
  static_assert(O_COL1 + NPV <= TMEM_COLS, "TMEM columns");
  static constexpr size_t PIECE = (size_t)(D / 4 + 1) * BM;                 // float4 of one piece of one stream: O, then {m, l, l exact, 128 + V's reference or 0: no O}
};

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// 2^e for e <= 127, as far down as there are subnormal numbers.
__device__ __forceinline__ float pow2i(int e) {
  return __uint_as_float((uint32_t)(max(e < -126 ? e + 64 : e, -126) + 127) << 23) * (e < -126 ? 0x1p-64f : 1.f);
}

// Weights of the key columns [C0, C1) of a tile as in the clip kernel, packed to fp16.
template <int C0, int C1, bool LSE>
__device__ __forceinline__ void take_weights_f16(const uint32_t (&s)[BN], uint32_t (&pk)[BN / 2], float2& la, float2 sc2, float2 mneg) {
#pragma unroll
  for (int c = C0; c < C1; c += 4) {
    float2 e0 = __ffma2_rn(make_float2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), sc2, mneg);
    float2 e1 = __ffma2_rn(make_float2(__uint_as_float(s[c + 2]), __uint_as_float(s[c + 3])), sc2, mneg);
    e0.x = ex2(e0.x); e0.y = ex2(e0.y);
    e1.x = ex2(e1.x); e1.y = ex2(e1.y);
    pk[c / 2] = pack_f16(e0.x, e0.y);
    pk[c / 2 + 1] = pack_f16(e1.x, e1.y);
    if (LSE) la = __fadd2_rn(la, __fadd2_rn(e0, e1));
  }
}
__device__ __forceinline__ void sts128(uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void sts64(uint32_t at, uint32_t x, uint32_t y) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(x), "r"(y) : "memory");
}

// Which 16-byte chunk of codes a thread of the widening warps takes in pass p: eight neighbouring lanes read and write eight
// different 16-byte columns of shared memory (rows r and r ^ 5 differ in both swizzles; nearly so at D = 96).
template <int D>
__device__ __forceinline__ void widen_place(int p, int warp, int lane, int& row, int& c) {
  const int five = (lane >> 2) & 1 ? 5 : 0;
  if (D == 128) {
    row = (p >> 1) * 32 + warp * 8 + ((((lane >> 4) & 1) | ((p & 1) << 1)) ^ five);
    c = ((lane >> 3) & 1) * 4 + (lane & 3);
  } else if (D == 64) {
    row = p * 32 + warp * 8 + (lane >> 2);
    c = lane & 3;
  } else if (p < 4) {
    row = p * 32 + warp * 8 + (((lane >> 3) & 3) ^ five);
    c = lane & 3;
  } else {
    const int i = lane >> 1;
    row = (p - 4) * 64 + warp * 16 + (((i & 3) << 1) | ((i >> 2) & 1) | (i & 8));
    c = 4 + (lane & 1);
  }
}

struct Maps { CUtensorMap q, k, v; };

template <int D, bool LSE>
__global__ void __launch_bounds__(kThreads, 1) rf_cache_chunk_kernel(const __grid_constant__ Maps maps, const __grid_constant__ RfCacheAttn a) {
  using C = Cfg<D>;
  constexpr uint32_t IDESC_HI = idesc_f8(BM, BN, 0), IDESC_LO = idesc_f8(BM, BN, 1), IDESC_PV = idesc_f16(BM, C::NPV, 1);
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - smem_u32(smem_raw));
  auto bar = [&](int slot) -> uint32_t { return base + C::BAR + 8u * slot; };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(base_ptr + C::MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + C::MISC + 8);
  int* items = reinterpret_cast<int*>(base_ptr + C::ITEM);
  volatile uint32_t* records = reinterpret_cast<volatile uint32_t*>(base_ptr + C::RECORD);
  StretchScratch<ChunkItem>* scratch = reinterpret_cast<StretchScratch<ChunkItem>*>(base_ptr + C::SCRATCH);
  volatile int* refs = reinterpret_cast<volatile int*>(base_ptr + C::REF);
  volatile uint32_t* flags = reinterpret_cast<volatile uint32_t*>(base_ptr + C::FLAGS);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    mbar_init(bar(C::B_Q), 4);
    mbar_init(bar(C::B_QE), 1);
    mbar_init(bar(C::B_QR), 1);
#pragma unroll 1
    for (int s = 0; s < C::NK; ++s) { mbar_init(bar(C::B_KF + s), 1); mbar_init(bar(C::B_KE + s), 1); }
#pragma unroll 1
    for (int s = 0; s < C::NV; ++s) { mbar_init(bar(C::B_VF + s), 4); mbar_init(bar(C::B_VE + s), 1); }
    for (int j = 0; j < 2; ++j) {
      mbar_init(bar(C::B_SF + j), 2);                        // the scores' products, and the MMA thread, which has written V's reference
      for (int p = 0; p < C::PARTS; ++p) mbar_init(bar(C::B_PF + j * C::PARTS + p), 4);
      mbar_init(bar(C::B_OF + j), 1);
      mbar_init(bar(C::B_SE + j), 4);
    }
#pragma unroll 1
    for (int i = 0; i < kItemSlots; ++i) { mbar_init(bar(C::B_IF + i), 1); mbar_init(bar(C::B_IE + i), kItemReaders); }
#pragma unroll 1
    for (int i = 0; i < C::NS; ++i) { mbar_init(bar(C::B_CF + i), 1); mbar_init(bar(C::B_CE + i), 4); }
    *abort_flag = 0;
    mbar_init_fence();
  }
#pragma unroll 1
  for (int i = tid; i < C::NV * BN * 2; i += kThreads) {   // the 16 columns behind V's: one, then zeros
    const int v = i / (BN * 2), row = i / 2 % BN, c = i % 2;
    *reinterpret_cast<uint4*>(base_ptr + C::V0 + v * C::VTILE + C::VLOAD + C::vchunk(row, c)) = make_uint4(c == 0 ? 0x3c00u : 0u, 0u, 0u, 0u);
  }
  fence_proxy_async_smem();
  if (warp == kPagesWarp) {
    if (lane == 0) { prefetch_tmap(&maps.q); prefetch_tmap(&maps.k); prefetch_tmap(&maps.v); }
    __syncwarp();
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), C::TMEM_COLS);
  }
  rf_grid_wait();
  tc_fence_before();
  const Stretch st = rf_cache_attn::stretch<ChunkPlaces, kThreads>(a, scratch);   // (has barriers)
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const WaitCtx wc{abort_flag, a.dev_status};
  if (tid == 0) {
    int32_t* head = reinterpret_cast<int32_t*>(a.ws) + blockIdx.x * kHeadWords;
    head[0] = st.item;
    head[3] = st.cuts;
  }

  if (warp >= kWidenWarp) {
    RF_REGS_WIDEN();
    // ------------------------------------------------------------ Q in two parts, V's codes to fp16
    const int w = warp - kWidenWarp;
    // An item's rows, kLanes neighbouring lanes a row (16 bytes each), in place: a warp has read its rows before it writes their parts.  (What
    // the parts of rows past the last hold does not matter: no such row is stored.)
    auto split_q = [&](int slot, int rows) {
      // Four steps' rows together, as a step is a chain of shuffles and conversions (9050 cycles for 256 rows two at a time and by way of
      // fp32, 5120 so); rows' maxima in pairs.  In fp16 a scaled row and what hi leaves of it are exact down to 2^-24.
      constexpr int kLanes = D == 64 ? 8 : 16, kRowsAtOnce = 32 / kLanes, kTogether = 4;
      const int c = lane % kLanes;
#pragma unroll 1
      for (int s0 = w * kRowsAtOnce + lane / kLanes; s0 - lane / kLanes < rows; s0 += 4 * kRowsAtOnce * kTogether) {
        uint4 v[kTogether];
        uint32_t most[kTogether / 2];         // two rows' largest magnitudes, as bf16 bits
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
          const int j = (s0 + k * 4 * kRowsAtOnce) >> 7, row = (s0 + k * 4 * kRowsAtOnce) & 127;
          const uint32_t at = D == 64 ? C::RAW + j * 128 * 128 : C::Q + (2 * j + (c >> 3)) * C::TILE;
          v[k] = c < D / 8 ? *reinterpret_cast<const uint4*>(base_ptr + at + row * 128 + (((c & 7) ^ (row & 7)) << 4)) : make_uint4(0u, 0u, 0u, 0u);
          const uint32_t m = __vmaxu2(__vmaxu2(v[k].x & 0x7fff7fffu, v[k].y & 0x7fff7fffu), __vmaxu2(v[k].z & 0x7fff7fffu, v[k].w & 0x7fff7fffu));
          const uint32_t one = max(m >> 16, m & 0xffffu);
          most[k / 2] = k & 1 ? most[k / 2] | one << 16 : one;
        }
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) {
#pragma unroll
          for (int k = 0; k < kTogether / 2; ++k) most[k] = __vmaxu2(most[k], __shfl_xor_sync(0xffffffffu, most[k], d));
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < kTogether; ++k) {
          const int rr = s0 + k * 4 * kRowsAtOnce, row = rr & 127;
          const uint32_t* u = &v[k].x;
          const uint32_t top = k & 1 ? most[k / 2] >> 16 : most[k / 2] & 0xffffu;
          // times 2^e the largest lies in (224, 448]; a row with a value that is not finite gets that in its scale, so that its scores have it
          const int e = top == 0u ? 0 : min(8 - ((int)(top >> 7) - 127) - ((top & 127u) > 96u ? 1 : 0), 126);
          const float up = __uint_as_float((uint32_t)(e + 127) << 23);
          if (c == 0) base_ptr[C::ROWEXP + slot * kRows + rr] = top >= 0x7f80u ? 255 : (uint8_t)(127 - e);
          uint32_t hi[2] = {}, lo[2] = {};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t q2 = pack_f16(__uint_as_float(u[i] << 16) * up, __uint_as_float(u[i] & 0xffff0000u) * up);
            const __half2_raw q2h = *reinterpret_cast<const __half2_raw*>(&q2);
            const uint32_t h2 = __nv_cvt_halfraw2_to_fp8x2(q2h, __NV_SATFINITE, __NV_E4M3);
            const __half2 rest = __hsub2(*reinterpret_cast<const __half2*>(&q2), __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)h2, __NV_E4M3)));
            const uint32_t l2 = __nv_cvt_halfraw2_to_fp8x2(*reinterpret_cast<const __half2_raw*>(&rest), __NV_SATFINITE, __NV_E5M2);
            hi[i / 2] |= h2 << (16 * (i & 1));
            lo[i / 2] |= l2 << (16 * (i & 1));
          }
          if (c < D / 8) {
            const uint32_t at = base + C::Q + (rr >> 7) * 2 * C::TILE + C::qchunk(row, c >> 1) + (c & 1) * 8;
            sts64(at, hi[0], hi[1]);
            sts64(at + C::TILE, lo[0], lo[1]);
          }
        }
      }
    };
    int nq = 0;                               // items with tiles so far
#pragma unroll 1
    for (int u = 0;; ++u) {
      const int cs = u % C::NS, vs = u % C::NV;
      if (!__all_sync(0xffffffffu, mbar_wait(bar(C::B_CF + cs), (u / C::NS) & 1, wc))) break;
      volatile const uint32_t* r = records + cs * 4;
      const uint32_t f = r[0], factor = r[1];
      const int valid = (int)r[2];                            // tokens of the page; behind them may lie codes of no number
      if (!(f & kMore)) break;
      if (f & kFirst) {
        if (!__all_sync(0xffffffffu, mbar_wait(bar(C::B_QR), nq & 1, wc))) break;
        ++nq;
        split_q((int)r[3], min(kRows, a.u.rows - items[(int)r[3] * kItemWords + 1]));
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::B_Q));
      }
      if (u >= C::NV && !__all_sync(0xffffffffu, mbar_wait(bar(C::B_VE + vs), ((u / C::NV) - 1) & 1, wc))) break;
      const uint8_t* from = base_ptr + C::VS0 + cs * C::TILE;
      const uint32_t to = base + C::V0 + vs * C::VTILE;
#pragma unroll kUnroll
      for (int p = 0; p < D / 16; ++p) {
        int row, c;
        widen_place<D>(p, w, lane, row, c);
        uint4 x = *reinterpret_cast<const uint4*>(from + C::qchunk(row, c));
        if (row >= valid) x = make_uint4(0u, 0u, 0u, 0u);
        const uint32_t* in = &x.x;
        uint32_t y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[2 * i] = mul_f16x2(widen_low(in[i]), factor);
          y[2 * i + 1] = mul_f16x2(widen_high(in[i]), factor);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
          sts128(to + (2 * c / (C::VBOX / 8)) * C::VBLK + C::vchunk(row, (2 * c + i) % (C::VBOX / 8)), y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) { mbar_arrive(bar(C::B_CE + cs)); mbar_arrive(bar(C::B_VF + vs)); }
    }
  } else if (warp >= kPagesWarp) {
    RF_REGS_CONTROL();
    if (warp == kPagesWarp) {
      // ------------------------------------------------------------ pages
      int* win = reinterpret_cast<int*>(base_ptr + C::WINDOW);
      int no = 0, u = 0, nq = 0;          // items published, tiles published, Q fetched
      long long at = st.at;
      int item = st.item;
      bool ok = true;
#pragma unroll 1
      for (long long pos = st.lo; pos < st.hi && ok; ++item) {
        const ChunkItem s = item == st.item ? scratch->info : chunk_item(a, item);
        const CacheItem it = s.it;
        if (!s.there) continue;
        const int n = max(s.n0, s.n1), begin = (int)(pos - at), end = (int)min((long long)n, st.hi - at);
        at += n + kItemPlaces;
        pos = min(at, st.hi);
        if (begin > 0 && begin >= n) continue;            // only the places of the item's end
        int b0, b1, e0, e1;
        if (a.count == nullptr) {       // the streams keep step: they share their tiles
          b0 = min(begin, s.n0); e0 = min(end, s.n0);
          b1 = min(begin, s.n1); e1 = min(end, s.n1);
        } else {
          b0 = (int)((long long)s.n0 * begin / n); e0 = (int)((long long)s.n0 * end / n);
          b1 = (int)((long long)s.n1 * begin / n); e1 = (int)((long long)s.n1 * end / n);
        }
        const int pages = rf_pages(it.len), slot = no % kItemSlots;
        if (no >= kItemSlots) ok = __all_sync(0xffffffffu, mbar_wait_long(bar(C::B_IE + slot), ((no / kItemSlots) - 1) & 1, wc, end - begin));
        if (!ok) break;
        if (lane == 0) {
          int* w = items + slot * kItemWords;
          w[0] = it.bh; w[1] = it.r0; w[2] = it.len; w[3] = it.q_len; w[4] = pages; w[5] = e0 - b0; w[6] = e1 - b1; w[7] = b0; w[8] = b1;
          w[10] = it.origin;
          w[9] = (begin > 0 ? kHeadPiece : 0) | (end < n && begin == 0 ? kTailPiece : 0);
          mbar_arrive(bar(C::B_IF + slot));
        }
        ++no;
        if (e0 == b0 && e1 == b1) continue;                    // sees nothing, or lists nothing here
        bool first = true;
        int ref = 0, top0 = -128, top1 = -128;                 // V's reference; the highest that it has been for either stream's rows
        const int32_t* l0 = a.count != nullptr ? a.pages + ((size_t)it.bh * a.u.n_q + it.r0 / kPage) * a.n_k : nullptr;
        const int32_t* l1 = l0 != nullptr && it.r0 / kPage + 1 < a.u.n_q ? l0 + a.n_k : l0;
        int i0 = b0, i1 = b1;
#pragma unroll 1
        while ((i0 < e0 || i1 < e1) && ok) {
          // a batch of the union: entries past the sequence count as page `pages`, which no row sees
          int m0 = 0x7fffffff, m1 = 0x7fffffff;
          if (lane < kBatch) {
            if (i0 + lane < e0) m0 = l0 != nullptr ? l0[i0 + lane] : i0 + lane;
            if (i1 + lane < e1) m1 = l1 != nullptr ? l1[i1 + lane] : i1 + lane;
            if (i0 + lane < e0 && (m0 < 0 || m0 >= pages)) { m0 = pages; rf_report(a.dev_status, RF_ERR_INVALID_ARG); }
            if (i1 + lane < e1 && (m1 < 0 || m1 >= pages)) { m1 = pages; rf_report(a.dev_status, RF_ERR_INVALID_ARG); }
            win[lane] = m0;
            win[kBatch + lane] = m1;
          }
          __syncwarp();
          int take0 = 0, take1 = 0, cnt = 0;
          if (lane == 0) {
#pragma unroll 1
            for (; cnt < kBatch; ++cnt) {
              const int h0 = take0 < kBatch ? win[take0] : 0x7fffffff, h1 = take1 < kBatch ? win[kBatch + take1] : 0x7fffffff;
              const int h = min(h0, h1);
              if (h == 0x7fffffff) break;
              win[2 * kBatch + cnt] = h;
              win[3 * kBatch + cnt] = (h0 == h ? 1 : 0) | (h1 == h ? 2 : 0);
              take0 += h0 == h;
              take1 += h1 == h;
            }
          }
          __syncwarp();
          take0 = __shfl_sync(0xffffffffu, take0, 0);
          take1 = __shfl_sync(0xffffffffu, take1, 0);
          cnt = __shfl_sync(0xffffffffu, cnt, 0);
          i0 += take0;
          i1 += take1;
          uint32_t row = 0, f = 0;
          int vexp = -128, valid = 0;
          if (lane < cnt) {
            const int page = win[2 * kBatch + lane];
            f = (uint32_t)win[3 * kBatch + lane] | kMore;
            if (lane == cnt - 1 && i0 == e0 && i1 == e1) f |= kLast;
            if (lane == 0 && first) f |= kFirst;
            const int phys = rf_page(a.c, it.b, min(page, pages - 1), a.dev_status);   // (a page that no row sees: any will do)
            row = (uint32_t)phys * a.c.H + it.bh % a.c.H;
            vexp = min(max((int)((__float_as_uint(a.c.v_scale[row]) >> 23) & 255u) - 127, -100), 100);
            valid = min(max(it.len - page * kPage, 0), kPage);
          }
          // V's reference: the first tile's scale, and another's where that is too far off
          int mine_ref = 0;
#pragma unroll 1
          for (int i = 0; i < cnt; ++i) {
            const int e = __shfl_sync(0xffffffffu, vexp, i), on = (int)__shfl_sync(0xffffffffu, f, i);
            const int least = max(on & 1 ? top0 : -128, on & 2 ? top1 : -128) - kMostDown;
            if ((first && i == 0) || e > ref + kMostUp || e < ref + kLeastUp || ref < least) ref = max(e, least);
            if (on & 1) top0 = max(top0, ref);
            if (on & 2) top1 = max(top1, ref);
            if (lane == i) mine_ref = ref;
          }
          const int up = vexp - mine_ref;                          // 2^up as fp16; below 2^-15, or zero, at the least reference only
          const uint32_t half = up >= -14 ? (uint32_t)(up + 15) << 10 : up >= -24 ? 1u << (up + 24) : 0u;
          f |= (uint32_t)(mine_ref + 128) << 8;
          // the tiles one after the other, each by the lane that looked it up
#pragma unroll 1
          for (int i = 0; i < cnt && ok; ++i, ++u) {
            const int cs = u % C::NS, ks = u % C::NK;
            if (u >= C::NK) ok = __all_sync(0xffffffffu, mbar_wait(bar(C::B_KE + ks), ((u / C::NK) - 1) & 1, wc));
            if (ok && lane == i) {
              flags[ks] = f;
              mbar_expect_tx(bar(C::B_KF + ks), C::TILE);
              tma_load_3d(base + C::K0 + ks * C::TILE, &maps.k, 0, 0, (int)row, bar(C::B_KF + ks));
            }
            if (ok && first) {                                     // the item before has taken its last scores: its Q may go
              if (nq > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar(C::B_QE), (nq - 1) & 1, wc));
              if (ok && lane == 0) {
                constexpr uint32_t kBlock = 128 * 128;             // 128 rows of 64 bf16
                mbar_expect_tx(bar(C::B_QR), 2 * ((D + 63) / 64) * kBlock);
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                  for (int kb = 0; kb < (D + 63) / 64; ++kb)
                    tma_load_3d(base + (D == 64 ? C::RAW : C::Q) + (j * ((D + 63) / 64) + kb) * kBlock, &maps.q, kb * 64, it.r0 + j * BM, it.bh, bar(C::B_QR));
              }
              ++nq;
              first = false;
            }
            if (ok && u >= C::NS) ok = __all_sync(0xffffffffu, mbar_wait(bar(C::B_CE + cs), ((u / C::NS) - 1) & 1, wc));
            if (ok && lane == i) {
              volatile uint32_t* r = records + cs * 4;
              r[0] = f; r[1] = half * 0x10001u; r[2] = (uint32_t)valid; r[3] = slot;
              mbar_expect_tx(bar(C::B_CF + cs), C::TILE);
              tma_load_3d(base + C::VS0 + cs * C::TILE, &maps.v, 0, 0, (int)row, bar(C::B_CF + cs));
            }
          }
          __syncwarp();
        }
      }
      // the end, for the warps that walk tiles and for those that walk items
      const int cs = u % C::NS, slot = no % kItemSlots, ks = u % C::NK;
      if (u >= C::NK) mbar_wait(bar(C::B_KE + ks), ((u / C::NK) - 1) & 1, wc);
      if (u >= C::NS) mbar_wait(bar(C::B_CE + cs), ((u / C::NS) - 1) & 1, wc);
      if (no >= kItemSlots) mbar_wait_long(bar(C::B_IE + slot), ((no / kItemSlots) - 1) & 1, wc, (int)min(st.hi - st.lo, 1ll << 20));
      if (lane == 0) {
        records[cs * 4] = 0;
        mbar_arrive(bar(C::B_CF + cs));
        flags[ks] = 0;
        mbar_arrive(bar(C::B_KF + ks));
        items[slot * kItemWords] = -1;
        mbar_arrive(bar(C::B_IF + slot));
      }
    } else if (warp == kMmaWarp) {
      // ------------------------------------------------------------ MMA issuer
      if (C::S_EARLY ? lane == 0 : elect_one()) {
        constexpr uint32_t SW128 = (1024u >> 4) | (1u << 14) | (2u << 29), SW64 = (512u >> 4) | (1u << 14) | (4u << 29);   // stride of 8 rows, version, swizzle
        constexpr uint32_t DESC_HI = C::PITCH == 128 ? SW128 : SW64, DESC_HI_V = C::VBOX == 64 ? SW128 : SW64;
        constexpr uint32_t LO_KMAJOR = 1u << 16, LO_VMAJOR = (C::VBLK >> 4) << 16;
        auto desc = [](uint32_t lo) -> uint64_t { return ((uint64_t)DESC_HI << 32) | lo; };
        auto desc_v = [](uint32_t lo) -> uint64_t { return ((uint64_t)DESC_HI_V << 32) | lo; };
        const uint32_t q_lo = ((base + C::Q) >> 4) | LO_KMAJOR, k_lo = ((base + C::K0) >> 4) | LO_KMAJOR;
        const uint32_t v_lo = ((base + C::V0) >> 4) | LO_VMAJOR;
        auto issue_s = [&](int j, int ks, uint32_t rec) {
          refs[j] = (int)(rec >> 8) - 128;
          mbar_arrive(bar(C::B_SF + j));
          uint32_t a0 = q_lo + 2 * j * (C::TILE >> 4);
          const uint32_t b0 = k_lo + ks * (C::TILE >> 4);
          asm volatile("" : "+r"(a0));
          const uint32_t t_d = tmem_base + (j ? C::S_COL1 : C::S_COL0);
          mma_f8_c<false>(t_d, desc(a0), desc(b0), IDESC_HI);
#pragma unroll
          for (int k = 1; k < D / 32; ++k) mma_f8_c<true>(t_d, desc(a0 + k * 2), desc(b0 + k * 2), IDESC_HI);
#pragma unroll
          for (int k = 0; k < D / 32; ++k) mma_f8_c<true>(t_d, desc(a0 + (C::TILE >> 4) + k * 2), desc(b0 + k * 2), IDESC_LO);
          tc_commit(bar(C::B_SF + j));
        };
        auto issue_pv = [&](int j, int vs, uint32_t acc, uint32_t par) {
          const uint32_t b0 = v_lo + vs * (C::VTILE >> 4);
          const uint32_t t_p = tmem_base + (j ? C::P_COL1 : C::P_COL0), t_o = tmem_base + (j ? C::O_COL1 : C::O_COL0);
#pragma unroll
          for (int p = 0; p < C::PARTS; ++p) {
            mbar_wait(bar(C::B_PF + j * C::PARTS + p), par, wc);
            tc_fence_after();
#pragma unroll
            for (int k = C::cut(p) / 16; k < C::cut(p + 1) / 16; ++k) {
              if (k == 0) mma_ts(t_o, t_p, desc_v(b0), IDESC_PV, acc);
              else mma_ts_c<true>(t_o, t_p + k * 8, desc_v(b0 + k * (16 * C::VROW >> 4)), IDESC_PV);
            }
          }
          tc_commit(bar(C::B_OF + j));
        };
        uint32_t pv_par = 0, s_par = 3, acc = 0, nq = 0, cur = 0;
        auto s_free = [&](int j) {
          if (C::S_EARLY) mbar_wait(bar(C::B_SE + j), (s_par >> j) & 1, wc);
          if (C::S_SHARED) mbar_wait(bar(C::B_SE + (j ^ 1)), (s_par >> (j ^ 1)) & 1, wc);
          if (C::S_EARLY || C::S_SHARED) tc_fence_after();
          s_par ^= 1u << j;
        };
        // the next tile's flags, once its K is in place; nothing after an abandoned wait
        auto next = [&](int u) -> uint32_t {
          if (!mbar_wait(bar(C::B_KF + u % C::NK), (u / C::NK) & 1, wc)) return 0u;
          tc_fence_after();
          return flags[u % C::NK];
        };
        // the scores of an item's first tile, for both streams
        auto open = [&](uint32_t rec, int u) {
          mbar_wait(bar(C::B_Q), nq & 1, wc);
          ++nq;
          tc_fence_after();
#pragma unroll 1
          for (int j = 0; j < 2; ++j)
            if (rec & (1 << j)) { s_free(j); issue_s(j, u % C::NK, rec); }
          tc_commit(bar(C::B_KE + u % C::NK));
          if (rec & kLast) tc_commit(bar(C::B_QE));
        };
        cur = next(0);
        if (cur & kMore) open(cur, 0);
#pragma unroll 1
        for (int u = 0; cur & kMore; ++u) {
          const int vs = u % C::NV, ks = (u + 1) % C::NK;
          uint32_t nxt = 0;
          if (cur & kLast) {
            if (!mbar_wait(bar(C::B_VF + vs), (u / C::NV) & 1, wc)) break;
            tc_fence_after();
#pragma unroll 1
            for (int j = 0; j < 2; ++j) {
              if (cur & (1 << j)) {
                issue_pv(j, vs, (acc >> j) & 1, (pv_par >> j) & 1);
                pv_par ^= 1u << j;
              }
            }
            tc_commit(bar(C::B_VE + vs));
            acc = 0;
            nxt = next(u + 1);
            if (nxt & kMore) open(nxt, u + 1);
          } else {
            nxt = next(u + 1);
            if (!(nxt & kMore)) break;
            if (!mbar_wait(bar(C::B_VF + vs), (u / C::NV) & 1, wc)) break;
            tc_fence_after();
            if constexpr (C::S_EARLY) {
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                if (nxt & (1 << j)) { s_free(j); issue_s(j, ks, nxt); }
                if (cur & (1 << j)) {
                  issue_pv(j, vs, (acc >> j) & 1, (pv_par >> j) & 1);
                  acc |= 1u << j;
                  pv_par ^= 1u << j;
                }
              }
            } else {
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                if (cur & (1 << j)) {
                  issue_pv(j, vs, (acc >> j) & 1, (pv_par >> j) & 1);
                  acc |= 1u << j;
                  pv_par ^= 1u << j;
                }
                if (nxt & (1 << j)) { s_free(j); issue_s(j, ks, nxt); }
              }
            }
            tc_commit(bar(C::B_KE + ks));
            tc_commit(bar(C::B_VE + vs));
            if (nxt & kLast) tc_commit(bar(C::B_QE));
          }
          cur = nxt;
        }
      }
    }
  } else {
    RF_REGS_SOFTMAX();
    // ------------------------------------------------------------ softmax + epilogue, one thread per query row (as in the clip kernel)
    const int j = warp >> 2, row_in_tile = tid & 127;
    const uint32_t lane_sel = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem_base + lane_sel + (j ? C::S_COL1 : C::S_COL0);
    const uint32_t t_o = tmem_base + lane_sel + (j ? C::O_COL1 : C::O_COL0);
    const float sc = a.scale_log2;
    uint32_t done = 0;
    int waited = 0;
#pragma unroll 1
    for (int item = 0;; ++item) {
      const int slot = item % kItemSlots;
      const int* iw = items + slot * kItemWords;
      if (!__all_sync(0xffffffffu, mbar_wait_long(bar(C::B_IF + slot), (item / kItemSlots) & 1, wc, waited))) break;
      if (iw[0] < 0) break;
      const int n = iw[5 + j], begin = iw[7 + j], end = begin + n, pages = iw[4];
      waited = iw[5] + iw[6];
      const int r = iw[1] + j * BM + row_in_tile;
      int sees = 0;                                       // keys that this row sees; none if it is padding
      if (r < a.u.rows && r % a.u.M < iw[3]) sees = rf_row_sees(a.u.causal, iw[10], iw[2], iw[3], r % a.u.M);
      const int32_t* list = a.count != nullptr ? a.pages + ((size_t)iw[0] * a.u.n_q + min(iw[1] / kPage + j, a.u.n_q - 1)) * a.n_k : nullptr;
      float m_run = -INFINITY, l_run = 0.f, l_exact = 0.f;
      int ref_run = 0;                                    // O is in units of 2^ref_run
      // The factor of a tile's scores holds the page's scale: the page is looked up two tiles ahead, its scale one.
      const int32_t* table = a.c.table + (size_t)(iw[0] / a.c.H) * a.c.max_pages;
      const float* k_scale = a.c.k_scale + iw[0] % a.c.H;
      auto page_of = [&](int t) -> int {
        const int p = list != nullptr ? list[t] : t;
        return p < 0 || p >= pages ? pages : p;
      };
      auto place_of = [&](int page) -> int { return min(max(table[min(page, pages - 1)], 0), a.c.n_pages - 1); };
      float row_scale = sc, ks_next = 0.f;
      int page_next = 0, place_next = 0;
      if (n > 0) {
        page_next = page_of(begin);
        ks_next = k_scale[(size_t)place_of(page_next) * a.c.H];
        if (n > 1) place_next = place_of(page_of(begin + 1));
      }
      if (n > 0) {
        // The rows' exponents are there once this stream's first scores are: the MMA thread has waited for Q before it issues them.  (B_Q itself
        // must not be waited for here.  Nothing holds an item's Q back until these warps have seen the item's before it, so its one-bit parity could
        // come round under a warp that is late.  The scores' barrier cannot: its next phase wants this warp's weights.)
        mbar_wait(bar(C::B_SF + j), done & 1, wc);
        const uint32_t e = base_ptr[C::ROWEXP + slot * kRows + j * BM + row_in_tile];
        row_scale *= __uint_as_float(e == 255u ? 0x7fc00000u : e << 23);
      }
      bool opens = true;
#pragma unroll 1
      for (int t = begin; t < end; ++t, ++done, opens = false) {
        const int left = sees - page_next * kPage;        // keys of the tile that this row sees (page <= 2^23: no overflow)
        float sc = row_scale * ks_next;
        if (left <= 0 || sc < 1.1754944e-38f) sc = 1.1754944e-38f;   // (a masked score, -inf, times zero or NaN would be no number)
        if (t + 1 < end) {
          page_next = page_of(t + 1);
          ks_next = k_scale[(size_t)place_next * a.c.H];
          if (t + 2 < end) place_next = place_of(page_of(t + 2));
        }
        const bool partial = __any_sync(0xffffffffu, left < BN);
        mbar_wait(bar(C::B_SF + j), done & 1, wc);
        tc_fence_after();
        const int tile_ref = refs[j];
        uint32_t s[128];
        uint32_t l_tile;
        if constexpr (!C::S_EARLY) l_tile = tmem_ld1(t_o + D);
        load_scores(t_s, s);
        if constexpr (!C::S_EARLY) l_run = opens ? 0.f : l_run + __uint_as_float(l_tile);
        if constexpr (C::S_SHARED) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::B_SE + j));
        }
        if (partial) {
#pragma unroll
          for (int c = 0; c < BN; ++c)
            if (c >= left) s[c] = 0xff800000u;
        }
        if constexpr (C::S_EARLY) {
          float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
          for (int c = 0; c < 128; c += 4) {
            mx0 = fmaxf(mx0, fmaxf(__uint_as_float(s[c]), __uint_as_float(s[c + 1])));
            mx1 = fmaxf(mx1, fmaxf(__uint_as_float(s[c + 2]), __uint_as_float(s[c + 3])));
          }
          const float m_tile = fmaxf(mx0, mx1) * sc;
          const bool raise = m_tile > m_run + kRaise || (m_run == -INFINITY && m_tile > -INFINITY);
          const int ref = opens || m_tile > m_run - kNothing ? tile_ref : ref_run;
          const bool any_raise = __any_sync(0xffffffffu, raise || ref != ref_run);
          float alpha = 1.f;
          if (raise) {
            alpha = ex2(m_run - m_tile);
            m_run = m_tile;
            l_run *= alpha;
            if (LSE) l_exact *= alpha;
          }
          bool o_landed = opens;
          if (!opens && any_raise) {
            mbar_wait(bar(C::B_OF + j), (done - 1) & 1, wc);
            o_landed = true;
            rescale_o<D>(t_o, alpha * pow2i(ref_run - ref));
          }
          ref_run = ref;
          const float m_use = m_run == -INFINITY ? 0.f : m_run;
          const float2 sc2 = make_float2(sc, sc), mneg = make_float2(kTop - m_use, kTop - m_use);
          float2 la = make_float2(0.f, 0.f);
          uint32_t pk[64];
          take_weights_f16<0, BN, LSE>(s, pk, la, sc2, mneg);
          if (LSE) l_exact += la.x + la.y;
          if (!o_landed) mbar_wait(bar(C::B_OF + j), (done - 1) & 1, wc);
          tc_fence_after();
          l_tile = tmem_ld1(t_o + D);
          {
            const uint32_t t_p = tmem_base + lane_sel + (j ? C::P_COL1 : C::P_COL0);
            uint32_t(&p0)[32] = *reinterpret_cast<uint32_t(*)[32]>(&pk[0]);
            uint32_t(&p1)[32] = *reinterpret_cast<uint32_t(*)[32]>(&pk[32]);
            tmem_st32(t_p, p0);
            tmem_st32(t_p + 32, p1);
            tc_wait_ld();
            tmem_st1(t_o + D, 0u);
            tc_wait_st();
          }
          l_run = opens ? 0.f : l_run + __uint_as_float(l_tile) * alpha;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(C::B_PF + j));
          continue;
        }
        uint32_t pk[64];
        float2 la = make_float2(0.f, 0.f);
        const float2 sc2 = make_float2(sc, sc);
        float m_use = m_run == -INFINITY ? 0.f : m_run;
        take_weights_f16<0, kSpec, LSE>(s, pk, la, sc2, make_float2(kTop - m_use, kTop - m_use));
        float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
        for (int c = 0; c < 128; c += 4) {
          mx0 = fmaxf(mx0, fmaxf(__uint_as_float(s[c]), __uint_as_float(s[c + 1])));
          mx1 = fmaxf(mx1, fmaxf(__uint_as_float(s[c + 2]), __uint_as_float(s[c + 3])));
        }
        const float m_tile = fmaxf(mx0, mx1) * sc;
        const int ref = opens || m_tile > m_run - kNothing ? tile_ref : ref_run;
        if (__any_sync(0xffffffffu, m_tile > m_run + kRaise || ref != ref_run)) {
          float alpha = 1.f;
          if (m_tile > m_run + kRaiseMargin) {
            alpha = ex2(m_run - m_tile);
            m_run = m_tile;
            l_run *= alpha;
            if (LSE) l_exact *= alpha;
          }
          if (!opens) {
            mbar_wait(bar(C::B_OF + j), (done - 1) & 1, wc);
            rescale_o_call<D>(t_o, alpha * pow2i(ref_run - ref));
          }
          ref_run = ref;
          m_use = m_run == -INFINITY ? 0.f : m_run;
          la = make_float2(0.f, 0.f);
          take_weights_f16<0, kSpec, LSE>(s, pk, la, sc2, make_float2(kTop - m_use, kTop - m_use));
        }
        const uint32_t t_p = tmem_base + lane_sel + (j ? C::P_COL1 : C::P_COL0);
        const float2 mneg = make_float2(kTop - m_use, kTop - m_use);
        take_weights_f16<kSpec, 64, LSE>(s, pk, la, sc2, mneg);
        store_weights<0, 64>(t_p, pk);
        tmem_st1(t_o + D, 0u);
        take_weights_f16<64, 80, LSE>(s, pk, la, sc2, mneg);
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::B_PF + j * C::PARTS));
        take_weights_f16<80, BN, LSE>(s, pk, la, sc2, mneg);
        store_weights<64, BN>(t_p, pk);
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(C::B_PF + j * C::PARTS + 1));
        if (LSE) l_exact += la.x + la.y;
      }
      if (n > 0) {
        mbar_wait(bar(C::B_OF + j), (done - 1) & 1, wc);
        tc_fence_after();
        const uint32_t l_tile = tmem_ld1(t_o + D);
        tc_wait_ld();
        l_run += __uint_as_float(l_tile);
      }
      const int cut = iw[9];
      if (cut) {
        float4* mine = reinterpret_cast<float4*>(a.ws + head_floats(gridDim.x)) +
                       (((size_t)2 * blockIdx.x + (cut & kTailPiece ? 1 : 0)) * 2 + j) * C::PIECE + row_in_tile;
        if (n > 0) {
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t v[32];
            tmem_ld32(t_o + c * 32, v);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i)
              __stcg(mine + (c * 8 + i) * BM, make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]),
                                                          __uint_as_float(v[4 * i + 3])));
          }
        }
        __stcg(mine + (D / 4) * BM, make_float4(m_run, l_run, l_exact, n > 0 ? (float)(ref_run + 128) : 0.f));
      } else {
        const size_t at_row = (size_t)iw[0] * a.u.rows + min(r, a.u.rows - 1);
        const bool there = r < a.u.rows && r % a.u.M < iw[3] && rf_in_bounds(at_row, (unsigned long long)a.c.B * a.c.H * a.u.rows, a.dev_status);
        uint4* o = reinterpret_cast<uint4*>(a.o + at_row * D);
        const bool o32 = (reinterpret_cast<uintptr_t>(a.o) & 31u) == 0;
        const float inv = l_run == 0.f ? 0.f : pow2i(ref_run) / l_run;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          if (n > 0) {                                     // (the same for the whole warp)
            tmem_ld32(t_o + c * 32, v);
            tc_wait_ld();
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0u;
          }
          if (there) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = pack_bf16(__uint_as_float(v[2 * i]) * inv, __uint_as_float(v[2 * i + 1]) * inv);
            store_columns(o + c * 4, v, o32);
          }
        }
        if (LSE && there) a.lse[at_row] = (m_run - kTop + log2f(l_exact)) * 0.6931471805599453f;
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(C::B_IE + slot));
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == kPagesWarp) {
    if (*abort_flag) __nanosleep(20000);
    __syncwarp();
    tmem_dealloc(tmem_base, C::TMEM_COLS);
  }
}

// Joins the pieces of the items that the stretches cut (see rf_cache_join_kernel): a thread per row, blockIdx.y = stream and 16 columns.
template <int D, bool LSE>
__global__ void __launch_bounds__(BM) rf_cache_chunk_join_kernel(const __grid_constant__ RfCacheAttn a, int ctas) {
  using C = Cfg<D>;
  rf_grid_wait();
  const int x = blockIdx.x + 1, j = blockIdx.y / (D / 16), c0 = blockIdx.y % (D / 16) * 4;
  const int32_t* heads = reinterpret_cast<const int32_t*>(a.ws);
  const int32_t* mine = heads + x * kHeadWords;
  if (!mine[3]) return;
  if (mine[3 - kHeadWords] && mine[-kHeadWords] == mine[0]) return;
  __shared__ int last;
  const int n = rf_cache_attn::cuts_from(heads, x, ctas, &last);
  const CacheItem it = rf_cache_attn::cache_item<kRows>(a, mine[0]);
  const int row = it.r0 + j * BM + threadIdx.x;
  if (row >= a.u.rows || row % a.u.M >= it.q_len) return;
  const float4* pieces = reinterpret_cast<const float4*>(a.ws + head_floats(ctas)) + threadIdx.x;
  float m = -INFINITY, l = 0.f, lx = 0.f;
  int ref = -128;
  float4 acc[4] = {};
#pragma unroll 2
  for (int i = 0; i <= n; ++i) {
    const float4* at = pieces + ((i == 0 ? (size_t)2 * (x - 1) + 1 : (size_t)2 * (x + i - 1)) * 2 + j) * C::PIECE;
    const float4 st = __ldcg(at + (D / 4) * BM);
    float4 o[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = __ldcg(at + (c0 + k) * BM);
    if (st.w == 0.f || (st.x == -INFINITY && st.y == 0.f)) continue;   // walked no tile, so its O was never written, or saw nothing in them
    float keep = 1.f, w = 1.f;
    if (st.x > m) {
      keep = ex2(m - st.x);                             // (0 from -inf on)
      m = st.x;
    } else if (st.x > -INFINITY) {
      w = ex2(st.x - m);
    }
    l = l * keep + st.y * w;
    lx = lx * keep + st.z * w;
    if (w == 0.f) continue;                             // units count where there is something in them
    const int mine_ref = (int)st.w - 128, top = keep == 0.f ? mine_ref : max(ref, mine_ref);
    keep *= pow2i(min(ref - top, 0));
    w *= pow2i(mine_ref - top);
    ref = top;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      acc[k].x = acc[k].x * keep + o[k].x * w;
      acc[k].y = acc[k].y * keep + o[k].y * w;
      acc[k].z = acc[k].z * keep + o[k].z * w;
      acc[k].w = acc[k].w * keep + o[k].w * w;
    }
  }
  const float inv = l == 0.f ? 0.f : pow2i(ref) / l;
  uint32_t v[8];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = pack_bf16(acc[k].x * inv, acc[k].y * inv);
    v[2 * k + 1] = pack_bf16(acc[k].z * inv, acc[k].w * inv);
  }
  const size_t at_row = (size_t)it.bh * a.u.rows + row;
  if (!rf_in_bounds(at_row, (unsigned long long)a.c.B * a.c.H * a.u.rows, a.dev_status)) return;
  store_sector(reinterpret_cast<uint4*>(a.o + at_row * D) + c0 / 2, v, (reinterpret_cast<uintptr_t>(a.o) & 31u) == 0);
  if (LSE && c0 == 0) a.lse[at_row] = (m - kTop + log2f(lx)) * 0.6931471805599453f;
}

int chunk_ctas(const RfCache& c, const RfQueries& u) {
  const long long items = (long long)c.B * c.H * rf_cdiv(u.rows, kRows), most = items * c.max_pages;
  return (int)std::min<long long>(most, 148);
}

template <int D, bool LSE>
rf_status launch(const RfCacheAttn& a, cudaStream_t st) {
  using C = Cfg<D>;
  static bool configured[64] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return RF_ERR_CUDA;
  if (dev >= 0 && dev < 64 && !configured[dev]) {
    cudaFuncAttributes fa;
    if (cudaFuncGetAttributes(&fa, rf_cache_chunk_kernel<D, LSE>) != cudaSuccess) return RF_ERR_CUDA;
    // setmaxnreg.inc draws on what the launch owns: with less it would never be granted
    if (fa.numRegs * kThreads < 256 * kRegsSoftmax + 128 * kRegsControl + 128 * kRegsWiden) return RF_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(rf_cache_chunk_kernel<D, LSE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::ALLOC) != cudaSuccess)
      return RF_ERR_CUDA;
    configured[dev] = true;
  }
  Maps maps;
  if (!rf_encode_rows_map(&maps.q, a.u.q, D, a.u.rows, (size_t)D * 2, (size_t)a.u.rows * D * 2, a.c.B * a.c.H) || !rf_encode_pages_map(&maps.k, a.c.k, a.c) ||
      !rf_encode_pages_map(&maps.v, a.c.v, a.c))
    return RF_ERR_CUDA;
  const int ctas = chunk_ctas(a.c, a.u);
  if (rf_launch(rf_cache_chunk_kernel<D, LSE>, dim3(ctas), kThreads, C::ALLOC, st, maps, a) != cudaSuccess) return RF_ERR_CUDA;
  if (ctas == 1) return RF_OK;
  return rf_launch(rf_cache_chunk_join_kernel<D, LSE>, dim3(ctas - 1, 2 * (D / 16)), BM, 0, st, a, ctas) == cudaSuccess ? RF_OK : RF_ERR_CUDA;
}

}  // namespace

size_t rf_cache_chunk_ws_bytes(const RfCache& c, const RfQueries& u) {
  const int ctas = chunk_ctas(c, u);
  return head_floats(ctas) * sizeof(float) + (size_t)2 * ctas * 2 * (c.D / 4 + 1) * BM * sizeof(float4);
}

rf_status rf_launch_cache_chunk(const RfCacheAttn& a, cudaStream_t st) {
  const bool lse = a.lse != nullptr;
  switch (a.c.D) {
    case 64: return lse ? launch<64, true>(a, st) : launch<64, false>(a, st);
    case 96: return lse ? launch<96, true>(a, st) : launch<96, false>(a, st);
    case 128: return lse ? launch<128, true>(a, st) : launch<128, false>(a, st);
  }
  return RF_ERR_UNSUPPORTED;
}
