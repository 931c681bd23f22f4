// Rotary positions: tables of cosines and sines, and turning rows by them.  Both move bytes and are bound by HBM where there are many,
// by a launch where there are few.
#include "mes_attn.h"
#include "mes_rows.h"

namespace mes {
namespace {

// Row p of the table is e^(i p f).  A thread takes one frequency through kRun positions: it forms e^(i p f) once, for its first, and
// multiplies with e^(i f) from there on, all in 64 bits: the products' errors, kRun * 2^-52, stay far below fp32's 2^-24.  Bound by what it writes:
// 131072 positions of 128 dimensions, 67 MB in 12.5 us, 5.4 TB/s (6.8 is what clearing 2 GiB reaches).
constexpr int kRun = 16;
__global__ __launch_bounds__(256) void k_rotary_table(TableArgs a) {
  const int half = a.dims >> 1;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t first = id / half * kRun;
  const int i = (int)(id % half);
  if (first >= a.n_positions) return;
  const int n = (int)min((int64_t)kRun, a.n_positions - first);
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

// One workgroup per row (rows blockIdx, blockIdx + gridDim, ... where there are more than a launch has workgroups), a unit per thread.
// Gradients of 8192 tokens' rows (40 heads of 128, bf16): 172 MB in 33 to 35 us, 4.9 to 5.2 TB/s; 21 tokens as long as a launch.
template <class E>
__global__ __launch_bounds__(1024) void k_rotary(RotaryArgs a) {
  const int d = a.head_dim, per = d >> 4, units = (a.n_heads + a.n_kv_heads) * per, turned = a.dims >> 4;
  for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
    const int p = a.positions[t];
    const bool real = (unsigned)p < (unsigned)a.n_positions;
    if (!real && !a.fresh) continue;
    const float* row = a.table + (size_t)(real ? p : 0) * a.dims;
    for (int w = threadIdx.x; w < units; w += blockDim.x) {
      const int head = w / per, u = w % per;
      const bool key = head >= a.n_heads;
      const size_t h = (size_t)(key ? head - a.n_heads : head) * d;
      const E* in = static_cast<const E*>(key ? a.k : a.q) + (size_t)t * (key ? a.ld_k : a.ld_q) + h;
      E* out = static_cast<E*>(key ? a.k_out : a.q_out) + (size_t)t * (key ? a.ld_k_out : a.ld_q_out) + h;
      int i, j;
      chunks_of(u, a.dims, a.pairs, i, j);
      float x[8] = {}, y[8] = {};
      if (real) {
        load8(in + i, x);
        load8(in + j, y);
        if (u < turned) turn_unit(x, y, row, u, a.dims, a.pairs, a.sign);
      }
      store8(out + i, x);
      store8(out + j, y);
    }
  }
}

}  // namespace

hipError_t launch_rotary_table(const TableArgs& a, hipStream_t s) {
  const int64_t threads = (a.n_positions + kRun - 1) / kRun * (int64_t)(a.dims / 2);
  k_rotary_table<<<(unsigned)((threads + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_rotary(const RotaryArgs& a, bool fp32, hipStream_t s) {
  const int units = (a.n_heads + a.n_kv_heads) * (a.head_dim / 16), threads = std::min(1024, (units + 63) / 64 * 64);
  const unsigned grid = std::min((unsigned)a.T, 0xffffffffu / (unsigned)threads);   // a launch has up to 2^32 threads
  if (fp32) k_rotary<float><<<grid, threads, 0, s>>>(a);
  else k_rotary<uint16_t><<<grid, threads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace mes
