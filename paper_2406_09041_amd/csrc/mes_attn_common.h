// Device code that the attention kernels share.
#pragma once

#include "mes_attn.h"

namespace mes {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
// Weights are 2^(score - m) (scores in powers of two) with a running bound m of the row's scores.  Where a score passes it, it is raised to
// this much above the largest, so that the accumulators are rescaled a few times per row instead of at almost every tile; no weight is
// above 1 (a value of any size times its weight is finite), and the largest is at least 2^-kSlack, far from the ends of fp32 and bf16.
constexpr float kSlack = 8.0f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32; -inf gives 0

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  bf16x2 r;
  r[0] = (__bf16)a;
  r[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ float bf16_at(uint32_t w, int hi) { return __uint_as_float(hi ? w & 0xffff0000u : w << 16); }

// acc + lo(w) + hi(w)
__device__ __forceinline__ float add_pair(uint32_t w, float acc) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3f803f80u), acc, false);
}

// the value of lane l ^ 32, and of lane l ^ 16
__device__ __forceinline__ float other_half(float v) {
  const uint32_t u = __float_as_uint(v);
  const u32x2 r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
__device__ __forceinline__ float other_row16(float v) {
  const uint32_t u = __float_as_uint(v);
  const u32x2 r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 16) ? r[0] : r[1]);
}

// four e4m3 codes of a word times a power of two -> four bf16 (exact: a block's exponent costs nothing here)
__device__ __forceinline__ u32x2 widen4(uint32_t w, float power = 1.0f) {
  const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, false);
  const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, true);
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// The factor of scores that come from 8-bit codes holds the head's k_scale, which may have any sign.  Masked scores are -inf before it is
// multiplied in, and maxima are taken before it, so it has to be above 0: its sign, or all of it where it is 0 or NaN, goes to
// the query instead (exactly: bf16 times +-1, 0 or NaN).
__device__ __forceinline__ float factor_of_scores(float f) { return f > 0.0f ? f : f < 0.0f ? -f : 1.0f; }
template <class V, int N>
__device__ __forceinline__ void factor_to_query(V (&q)[N], float f) {
  if (f > 0.0f) return;
  const float by = f < 0.0f ? -1.0f : f;
#pragma unroll
  for (int c = 0; c < N; ++c) {
    u32x4 w = __builtin_bit_cast(u32x4, q[c]);
#pragma unroll
    for (int x = 0; x < 4; ++x) w[x] = pack2(bf16_at(w[x], 0) * by, bf16_at(w[x], 1) * by);
    q[c] = __builtin_bit_cast(V, w);
  }
}

// Over the lanes of a wavefront, without LDS.  scan: the sum up to and with the lane; max: of values that are not negative.
template <int CTRL, int ROWS>
__device__ __forceinline__ int from_below(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_scan(int v) {
  v += from_below<0x111, 0xf>(v);   // row_shr 1, 2, 4, 8: inside rows of 16
  v += from_below<0x112, 0xf>(v);
  v += from_below<0x114, 0xf>(v);
  v += from_below<0x118, 0xf>(v);
  v += from_below<0x142, 0xa>(v);   // row_bcast 15: row 0 to 1, 2 to 3
  v += from_below<0x143, 0xc>(v);   // row_bcast 31: rows 0 and 1 to 2 and 3
  return v;
}
__device__ __forceinline__ int wave_sum(int v) { return __builtin_amdgcn_readlane(wave_scan(v), 63); }
__device__ __forceinline__ int wave_max(int v) {
  v = max(v, from_below<0x111, 0xf>(v));
  v = max(v, from_below<0x112, 0xf>(v));
  v = max(v, from_below<0x114, 0xf>(v));
  v = max(v, from_below<0x118, 0xf>(v));
  v = max(v, from_below<0x142, 0xa>(v));
  v = max(v, from_below<0x143, 0xc>(v));
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

}  // namespace mes
