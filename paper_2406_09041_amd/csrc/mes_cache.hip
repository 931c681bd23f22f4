// Writing to the paged cache (rotary embedding of new queries and keys, keys and values to their pages) and copying its
// pages.  Both move bytes and are bound by HBM where there are many, by a launch where there are few.
#include "mes_attn.h"

namespace mes {
namespace {

constexpr int kAppendThreads = 256;

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

// x / scale to e4m3: a true division, so that the nearest code is that of the quotient; clamped before the conversion (which
// would make NaN of what is too large), NaN stays NaN.  0 stays 0 also where the scale is 0: a head that is
// always 0 has such a scale, and 0 / 0 would leave a NaN in the cache.
__device__ inline float to_grid(float x, float scale) {
  const float v = x == 0.0f && scale == 0.0f ? 0.0f : x / scale;
  return v > 448.0f ? 448.0f : v < -448.0f ? -448.0f : v;
}
__device__ inline uint32_t pack_e4m3(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

template <bool FP8>
__device__ inline void store8(void* base, size_t element, const float v[8], float scale) {
  if constexpr (FP8) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = to_grid(v[i], scale);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(base) + element) = make_uint2(pack_e4m3(t[0], t[1], t[2], t[3]), pack_e4m3(t[4], t[5], t[6], t[7]));
  } else {
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(base) + element) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  }
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

// Four prompts of 1024 tokens (32 query, 8 key / value heads of 128, bf16): 101 MB in 19.7 us, 5.1 TB/s; 256 single tokens 6 MB, as long as a launch.
//
// One workgroup per row.  A unit of work is 8 dimensions of the first half of a head and the 8 they turn with, so that q_out
// may be q: one thread reads both halves before it writes them.
template <bool FP8>
__global__ __launch_bounds__(kAppendThreads) void k_append(AppendArgs a) {
#pragma clang fp contract(off)   // products and sums are rounded one by one: the same bits as an elementwise program
  const int t = blockIdx.x;
  int s = t, behind = 1;                                   // sequence of the row, rows from it to the sequence's end
  if (a.q_offsets) {
    int lo = 0, hi = a.n_seqs;                             // first s with q_offsets[s + 1] > t
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (a.q_offsets[mid + 1] > t) hi = mid; else lo = mid + 1;
    }
    s = lo;
    if (s >= a.n_seqs || a.q_offsets[s] > t) s = -1;       // behind the last sequence
    else behind = a.q_offsets[s + 1] - t;
  }
  const int pos = s < 0 ? -1 : max(a.kv_len[s], 0) - behind;
  if (pos < 0 || pos >= a.capacity) {
    if (a.fresh)
      for (int i = threadIdx.x * 8; i < a.n_heads * a.head_dim; i += kAppendThreads * 8)
        *reinterpret_cast<uint4*>(a.q_out + (size_t)t * a.ld_q_out + i) = make_uint4(0, 0, 0, 0);
    return;
  }
  const int page = a.page_table[(size_t)s * a.table_pages + (pos >> a.page_shift)];
  const bool placed = (unsigned)page < (unsigned)a.n_pages;
  const int d = a.head_dim, half = d >> 1, per = half >> 3;   // per: units of a head
  const size_t slot = (size_t)(pos & ((1 << a.page_shift) - 1)) * d;
  const size_t head_step = (size_t)d << a.page_shift;
  const size_t page_at = ((size_t)a.layer * a.n_pages + (placed ? page : 0)) * a.n_kv_heads * head_step + slot;
  const float* turn = a.rotary ? a.rotary + (size_t)pos * d : nullptr;
  const int nq = a.q ? a.n_heads * per : 0, nk = a.n_kv_heads * per;
  for (int u = threadIdx.x; u < nq + 2 * nk; u += kAppendThreads) {
    const int w = u < nq ? u : u < nq + nk ? u - nq : u - nq - nk;
    const int h = w / per, i = (w % per) * 8;
    const uint16_t* row = u < nq ? a.q + (size_t)t * a.ld_q : u < nq + nk ? a.k + (size_t)t * a.ld_k : a.v + (size_t)t * a.ld_v;
    float x[8], y[8];
    load8(row + (size_t)h * d + i, x);
    load8(row + (size_t)h * d + half + i, y);
    if (u < nq + nk && turn) {
      float c[8], sn[8];
#pragma unroll
      for (int j = 0; j < 8; j += 4) {
        *reinterpret_cast<float4*>(c + j) = *reinterpret_cast<const float4*>(turn + i + j);
        *reinterpret_cast<float4*>(sn + j) = *reinterpret_cast<const float4*>(turn + half + i + j);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float p = x[j] * c[j], q = y[j] * sn[j], r = y[j] * c[j], o = x[j] * sn[j];
        x[j] = p - q;
        y[j] = r + o;
      }
    }
    if (u < nq) {
      store8<false>(a.q_out, (size_t)t * a.ld_q_out + (size_t)h * d + i, x, 1.0f);
      store8<false>(a.q_out, (size_t)t * a.ld_q_out + (size_t)h * d + half + i, y, 1.0f);
    } else if (placed) {
      const bool key = u < nq + nk;
      void* base = key ? a.k_cache : a.v_cache;
      const float scale = FP8 ? (key ? a.k_scale : a.v_scale)[(size_t)a.layer * a.n_kv_heads + h] : 1.0f;
      const size_t at = page_at + h * head_step;
      store8<FP8>(base, at + i, x, scale);
      store8<FP8>(base, at + half + i, y, scale);
    }
  }
}

// Pages are whole 16-byte words one behind the other; a workgroup copies up to kCopyBytes of one page of one layer of keys or
// values.  Where that is all of kCopyBytes, every load is in flight before the first store: 400 pages of 32 KiB in 32 layers of keys and values 360 us,
// 4.66 TB/s (4.84 is what a copy of 2 GiB reaches; a loop of one load and one store: 477 us).  Shorter pages, and the rest of longer ones, take
// that loop: 400 pages of 24, 16 and 8 KiB at 4.88, 4.81 and 4.65 TB/s, as more workgroups are there to wait side by side, but pages of 40 KiB
// at 3.2.
constexpr int kCopyThreads = 256, kCopyWords = 8, kCopyBytes = kCopyThreads * kCopyWords * 16;

struct CopyArgs {
  char *k, *v;
  size_t page_bytes, layer_bytes;
  int n_layers, parts;                 // parts: workgroups per page of a layer
  int32_t src[kCopyPairs], dst[kCopyPairs];
};

__global__ __launch_bounds__(kCopyThreads) void k_copy_pages(CopyArgs a) {
  const int part = blockIdx.x % a.parts, layer = (blockIdx.x / a.parts) % a.n_layers, pair = blockIdx.x / a.parts / a.n_layers;
  char* base = (blockIdx.y ? a.v : a.k) + layer * a.layer_bytes;
  const size_t at = (size_t)part * kCopyBytes + threadIdx.x * 16;
  const char* from = base + a.src[pair] * a.page_bytes;
  char* to = base + a.dst[pair] * a.page_bytes;
  constexpr int kStep = kCopyThreads * 16;
  uint4 w[kCopyWords];
  if ((size_t)(part + 1) * kCopyBytes <= a.page_bytes) {
#pragma unroll
    for (int i = 0; i < kCopyWords; ++i) w[i] = *reinterpret_cast<const uint4*>(from + at + i * kStep);
#pragma unroll
    for (int i = 0; i < kCopyWords; ++i) *reinterpret_cast<uint4*>(to + at + i * kStep) = w[i];
  } else {
    for (size_t x = at; x < a.page_bytes; x += kStep) *reinterpret_cast<uint4*>(to + x) = *reinterpret_cast<const uint4*>(from + x);
  }
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, int T, bool fp8, hipStream_t s) {
  if (fp8) k_append<true><<<T, kAppendThreads, 0, s>>>(a);
  else k_append<false><<<T, kAppendThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_copy_pages(const mes_kv& kv, const int32_t* src, const int32_t* dst, int n, hipStream_t s) {
  CopyArgs a;
  a.k = static_cast<char*>(kv.k);
  a.v = static_cast<char*>(kv.v);
  a.page_bytes = (size_t)kv.n_kv_heads * kv.page_tokens * kv.head_dim * (kv.dtype == MES_KV_E4M3 ? 1 : 2);
  a.layer_bytes = a.page_bytes * kv.n_pages;
  a.n_layers = kv.n_layers;
  a.parts = (int)((a.page_bytes + kCopyBytes - 1) / kCopyBytes);
  // a launch has up to 2^32 threads
  constexpr size_t kMostGrid = 0xffffffffu / kCopyThreads;
  const size_t per_pair = (size_t)a.parts * a.n_layers;
  if (per_pair > kMostGrid) return hipErrorInvalidValue;
  const int most = (int)std::min<size_t>(kCopyPairs, kMostGrid / per_pair);
  for (int i = 0; i < n; i += most) {
    const int m = std::min(most, n - i);
    for (int j = 0; j < m; ++j) {
      a.src[j] = src[i + j];
      a.dst[j] = dst[i + j];
    }
    k_copy_pages<<<dim3((unsigned)(per_pair * m), 2), kCopyThreads, 0, s>>>(a);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace mes
