// Rotary positions: tables of cosines and sines, and turning rows by them.  Both move bytes and are bound by HBM where there are many,
// by a launch where there are few.
#include "mes_attn.h"
#include "mes_rows.h"

namespace mes {
namespace {

// Row p of the table is e^(i p f).  A thread takes one frequency through `run` positions: it forms e^(i p f) once, for its first, and
// multiplies with e^(i f) from there on, all in 64 bits: the products' errors, run * 2^-52, stay far below fp32's 2^-24.
__global__ __launch_bounds__(256) void k_rotary_table(TableArgs a) {
  const int half = a.dims >> 1;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t first = id / half * a.run;
  const int i = (int)(id % half);
  if (first >= a.n_positions) return;
  const int n = (int)min((int64_t)a.run, a.n_positions - first);
  const double f = a.frequency[i];
  double c, s, cf, sf;
  sincos((double)first * f, &s, &c);
  sincos(f, &sf, &cf);
  c *= a.magnitude;
  s *= a.magnitude;
  float* out = a.table + first * a.dims + i;
  for (int p = 0; p < n; ++p) {
    out[0] = (float)c;
    out[half] = (float)s;
    out += a.dims;
    const double x = c * cf - s * sf;
    s = s * cf + c * sf;
    c = x;
  }
}

// One workgroup turns kRows rows, a thread the same unit of each, all of them on their way before the first is written.
template <class E, int kRows>
__global__ __launch_bounds__(1024) void k_rotary(RotaryArgs a) {
  const int d = a.head_dim, per = d >> 4, units = (a.n_heads + a.n_kv_heads) * per, turned = a.dims >> 4;
  const int t0 = blockIdx.x * kRows;
  int at[kRows];
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const int p = t0 + r < a.T ? a.positions[t0 + r] : -1;
    at[r] = (unsigned)p < (unsigned)a.n_positions ? p : -1;
  }
  for (int w = threadIdx.x; w < units; w += blockDim.x) {
    const int head = w / per, u = w % per;
    const bool key = head >= a.n_heads;
    const int h = key ? head - a.n_heads : head;
    const E* in = static_cast<const E*>(key ? a.k : a.q) + (size_t)h * d;
    E* out = static_cast<E*>(key ? a.k_out : a.q_out) + (size_t)h * d;
    const size_t ld = key ? a.ld_k : a.ld_q, ld_out = key ? a.ld_k_out : a.ld_q_out;
    int i, j;
    chunks_of(u, a.dims, a.pairs, i, j);
    float x[kRows][8], y[kRows][8];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[r][e] = y[r][e] = 0.0f;
      if (at[r] < 0) continue;
      load8(in + (t0 + r) * ld + i, x[r]);
      load8(in + (t0 + r) * ld + j, y[r]);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      if (t0 + r >= a.T || (at[r] < 0 && !a.fresh)) continue;
      if (u < turned && at[r] >= 0) turn_unit(x[r], y[r], a.table + (size_t)at[r] * a.dims, u, a.dims, a.pairs, a.sign);
      store8(out + (t0 + r) * ld_out + i, x[r]);
      store8(out + (t0 + r) * ld_out + j, y[r]);
    }
  }
}

}  // namespace

hipError_t launch_rotary_table(const TableArgs& args, hipStream_t s) {
  TableArgs a = args;
  const int half = a.dims / 2;
  a.run = 16;
  const int64_t threads = (a.n_positions + a.run - 1) / a.run * (int64_t)half;
  k_rotary_table<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_rotary(const RotaryArgs& a, bool fp32, hipStream_t s) {
  const int units = (a.n_heads + a.n_kv_heads) * (a.head_dim / 16), threads = std::min(1024, (units + 63) / 64 * 64);
  if (fp32) k_rotary<float, 1><<<a.T, threads, 0, s>>>(a);
  else k_rotary<uint16_t, 1><<<a.T, threads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mes
