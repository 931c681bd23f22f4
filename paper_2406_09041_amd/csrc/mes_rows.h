// Device code for rows of heads: 8 elements at a time, and turning them by rotary angles.
#pragma once

#include "mes_internal.h"

namespace mes {

__device__ inline float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ inline float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// two floats -> packed bf16, round to nearest even (v_cvt_pk_bf16_f32)
__device__ inline uint32_t pack_bf16(float a, float b) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  b2 r;
  r[0] = (__bf16)a;
  r[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, r);
}

__device__ inline void load8(const uint16_t* p, float v[8]) {
  const uint4 w = *reinterpret_cast<const uint4*>(p);
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_lo(u[i]);
    v[2 * i + 1] = bf16_hi(u[i]);
  }
}
__device__ inline void load8(const float* p, float v[8]) {
  *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(p);
  *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(p + 4);
}
__device__ inline void store8(uint16_t* p, const float v[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
}
__device__ inline void store8(float* p, const float v[8]) {
  *reinterpret_cast<float4*>(p) = *reinterpret_cast<const float4*>(v);
  *reinterpret_cast<float4*>(p + 4) = *reinterpret_cast<const float4*>(v + 4);
}

// A head's row is worked on in units of two chunks of 8 dimensions that turn with each other, so that one thread reads both before it writes
// either: in place is fine.  Unit u has the chunks a and b; units from dims / 16 on are not turned.
__device__ inline void chunks_of(int u, int dims, bool pairs, int& a, int& b) {
  const bool halves = !pairs && u < (dims >> 4);
  a = halves ? 8 * u : 16 * u;
  b = halves ? a + (dims >> 1) : a + 8;
}
// row: cosines and sines of the position, dims / 2 each.  sign: -1 turns back.
__device__ inline void turn_unit(float x[8], float y[8], const float* row, int u, int dims, bool pairs, float sign) {
#pragma clang fp contract(off)   // products and sums are rounded one by one: the same bits as an elementwise program
  float c[8], s[8];
  load8(row + 8 * u, c);
  load8(row + (dims >> 1) + 8 * u, s);
#pragma unroll
  for (int j = 0; j < 8; ++j) s[j] *= sign;
  if (pairs) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float& a = j < 4 ? x[2 * j] : y[2 * j - 8];
      float& b = j < 4 ? x[2 * j + 1] : y[2 * j - 7];
      const float p = a * c[j], q = b * s[j], r = b * c[j], o = a * s[j];
      a = p - q;
      b = r + o;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = x[j] * c[j], q = y[j] * s[j], r = y[j] * c[j], o = x[j] * s[j];
      x[j] = p - q;
      y[j] = r + o;
    }
  }
}

}  // namespace mes
