// The softmax warps' pieces that the tcgen05 attention kernels share: one thread per query row, scores and O in TMEM.
#pragma once

#include "rf_attn_common.cuh"

namespace rf_attn {

// 16 and 32 bf16 columns of an output row.
__device__ __forceinline__ void store_sector(uint4* dst, const uint32_t* v, bool o32) {
  if (o32) {
    st_global_v8(dst, v);
  } else {
    dst[0] = make_uint4(v[0], v[1], v[2], v[3]);
    dst[1] = make_uint4(v[4], v[5], v[6], v[7]);
  }
}
__device__ __forceinline__ void store_columns(uint4* dst, const uint32_t* v, bool o32) {
  store_sector(dst, v, o32);
  store_sector(dst + 2, v + 8, o32);
}

// This thread's row of O times alpha (warp-collective).
__device__ __forceinline__ void rescale_columns(uint32_t t_o, float alpha) {
  uint32_t v[32];
  tmem_ld32(t_o, v);
  tc_wait_ld();
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * alpha);
  tmem_st32(t_o, v);
}
template <int D>
__device__ __forceinline__ void rescale_o(uint32_t t_o, float alpha) {
  tc_fence_after();
#pragma unroll
  for (int c = 0; c < D; c += 32) rescale_columns(t_o + c, alpha);
  tc_wait_st();
  tc_fence_before();
}
// The same out of line, for D = 96 / 128: rare as it is, the scores then stay in registers around it and the loop over the
// tiles is free of spills.  (At D = 64, inline, 16 bytes are spilt; out of line none, but 48 heads of 17 776 tokens took 5013 us
// instead of 4932 dense and 2676 instead of 2639 all Textural.)
template <int D>
__device__ __noinline__ void rescale_o_call(uint32_t t_o, float alpha) {
  tc_fence_after();
#pragma unroll 1
  for (int c = 0; c < D; c += 32) rescale_columns(t_o + c, alpha);
  tc_wait_st();
  tc_fence_before();
}

// This thread's row of scores, and the masked ones of a PARTIAL tile set to -inf.
__device__ __forceinline__ void load_scores(uint32_t t_s, uint32_t (&s)[BN]) {
  tmem_ld32(t_s, *reinterpret_cast<uint32_t(*)[32]>(&s[0]));
  tmem_ld32(t_s + 32, *reinterpret_cast<uint32_t(*)[32]>(&s[32]));
  tmem_ld32(t_s + 64, *reinterpret_cast<uint32_t(*)[32]>(&s[64]));
  tmem_ld32(t_s + 96, *reinterpret_cast<uint32_t(*)[32]>(&s[96]));
  tc_wait_ld();
}
__device__ __forceinline__ void mask_scores(const uint4* keep, uint32_t (&s)[BN]) {
  const uint4 kw = *keep;
  const uint32_t w[4] = {kw.x, kw.y, kw.z, kw.w};
#pragma unroll
  for (int c = 0; c < BN; ++c)
    if (!((w[c >> 5] >> (c & 31)) & 1u)) s[c] = 0xff800000u;  // -inf
}

// Weights of the key columns [C0, C1) of a tile: 2^(score * sc - m), packed to bf16; with LSE also their sum before rounding.
template <int C0, int C1, bool LSE>
__device__ __forceinline__ void take_weights(const uint32_t (&s)[BN], uint32_t (&pk)[BN / 2], float2& la, float2 sc2, float2 mneg) {
#pragma unroll
  for (int c = C0; c < C1; c += 4) {
    float2 e0 = __ffma2_rn(make_float2(__uint_as_float(s[c]), __uint_as_float(s[c + 1])), sc2, mneg);
    float2 e1 = __ffma2_rn(make_float2(__uint_as_float(s[c + 2]), __uint_as_float(s[c + 3])), sc2, mneg);
    e0.x = ex2(e0.x); e0.y = ex2(e0.y);
    e1.x = ex2(e1.x); e1.y = ex2(e1.y);
    pk[c / 2] = pack_bf16(e0.x, e0.y);
    pk[c / 2 + 1] = pack_bf16(e1.x, e1.y);
    if (LSE) la = __fadd2_rn(la, __fadd2_rn(e0, e1));
  }
}

// The packed weights of the key columns [C0, C1) into P.  Eight registers at a time: longer stores want that many consecutive
// registers, which costs moves (24 heads, 8448 tokens, dense, D = 128: 1153 kcycles a call with 32, 1112 with 16, 1108 with 8).
template <int C0, int C1>
__device__ __forceinline__ void store_weights(uint32_t t_p, const uint32_t (&pk)[BN / 2]) {
#pragma unroll
  for (int c = C0 / 2; c < C1 / 2; c += 8) tmem_st8(t_p + c, *reinterpret_cast<const uint32_t(*)[8]>(&pk[c]));
}

}  // namespace rf_attn
