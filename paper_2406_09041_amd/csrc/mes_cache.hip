// Writing to the paged cache (rotary embedding of new queries and keys, keys and values to their pages) and copying its
// pages.  Both move bytes and are bound by HBM where there are many, by a launch where there are few.
#include "mes_attn.h"
#include "mes_place.h"
#include "mes_rows.h"

namespace mes {
namespace {

constexpr int kAppendThreads = 256;

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

// 8 values times a power of two -> codes, what is past the limit to the limit, NaN stays NaN
__device__ inline uint2 codes8(const float v[8], float by, float limit) {
  float t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = v[i] * by;
    t[i] = x > limit ? limit : x < -limit ? -limit : x;
  }
  return make_uint2(pack_e4m3(t[0], t[1], t[2], t[3]), pack_e4m3(t[4], t[5], t[6], t[7]));
}
template <int I>
__device__ inline float code_at(uint32_t w) { return __builtin_amdgcn_cvt_f32_fp8(w, I); }
// four codes to those of a larger exponent
__device__ inline uint32_t scaled4(uint32_t w, float by) { return pack_e4m3(code_at<0>(w) * by, code_at<1>(w) * by, code_at<2>(w) * by, code_at<3>(w) * by); }
// two codes of a word times a power of two -> bf16
template <bool HIGH>
__device__ inline uint32_t widen2(uint32_t w, float power) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, power, HIGH)); }

template <bool FP8>
__device__ inline void put8(void* base, size_t element, const float v[8], float scale) {
  if constexpr (FP8) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = to_grid(v[i], scale);
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(base) + element) = make_uint2(pack_e4m3(t[0], t[1], t[2], t[3]), pack_e4m3(t[4], t[5], t[6], t[7]));
  } else {
    store8(static_cast<uint16_t*>(base) + element, v);
  }
}

// Four prompts of 1024 tokens (32 query, 8 key / value heads of 128, bf16): 101 MB in 19.7 us, 5.1 TB/s; 256 single tokens 6 MB, as long as a launch.
//
// The first s with offsets[s + 1] > t, n where there is none; t is the same in all 64 lanes.  Two dependent loads (one up to 64 sequences), where
// a search by halves would take one for each.
__device__ __forceinline__ int sequence_of(const int32_t* offsets, int n, int t) {
  if (n == 0) return 0;
  const int lane = threadIdx.x & 63, step = (n + 63) >> 6;
  const int first = __popcll(__ballot(offsets[min((lane + 1) * step, n)] <= t)) * step;
  if (step == 1 || first >= n) return min(first, n);
  return min(first + __popcll(__ballot(lane < step && offsets[min(first + lane + 1, n)] <= t)), n);
}
// s: the row's sequence, by sequence_of
template <class A>
__device__ __forceinline__ Place place_in(const A& a, int t, int s) {
  if (s >= a.n_seqs) return kNoPlace;
  return place_of_row(s, a.q_offsets ? a.q_offsets[s] : t, a.q_offsets ? a.q_offsets[s + 1] : t + 1, a.kv_len[s], a.capacity, t, a.T);
}
template <class A>
__device__ __forceinline__ Place place_of(const A& a, int t) { return place_in(a, t, a.q_offsets ? sequence_of(a.q_offsets, a.n_seqs, t) : t); }

// q's part of a row: turned, rounded once, to q_out; 0 where the row has no place and nothing is there yet
__device__ __forceinline__ void append_queries(const AppendArgs& a, int t, const float* turn, bool real) {
  const int d = a.head_dim, per = d >> 4, units = a.n_heads * per;
  if (!real) {
    if (a.fresh)
      for (int i = threadIdx.x * 8; i < a.n_heads * d; i += kAppendThreads * 8) *reinterpret_cast<uint4*>(a.q_out + (size_t)t * a.ld_q_out + i) = make_uint4(0, 0, 0, 0);
    return;
  }
  for (int w = threadIdx.x; w < units; w += kAppendThreads) {
    const int h = w / per, u = w % per;
    int i, j;
    chunks_of(u, a.dims, a.pairs, i, j);
    float x[8], y[8];
    load8(a.q + (size_t)t * a.ld_q + (size_t)h * d + i, x);
    load8(a.q + (size_t)t * a.ld_q + (size_t)h * d + j, y);
    if (u < a.dims >> 4) turn_unit(x, y, turn, u, a.dims, a.pairs, 1.0f);
    store8(a.q_out + (size_t)t * a.ld_q_out + (size_t)h * d + i, x);
    store8(a.q_out + (size_t)t * a.ld_q_out + (size_t)h * d + j, y);
  }
}

// One workgroup per row.  A unit of work is 8 dimensions of the first half of a head and the 8 they turn with, so that q_out
// may be q: one thread reads both halves before it writes them.
template <bool FP8>
__global__ __launch_bounds__(kAppendThreads) void k_append(AppendArgs a) {
  const int t = blockIdx.x;
  const Place at = place_of(a, t);
  const int s = at.seq, pos = at.pos;
  if (pos < 0 || pos >= a.capacity) return append_queries(a, t, nullptr, false);
  const int page = a.page_table[(size_t)s * a.table_pages + (pos >> a.page_shift)];
  const bool placed = (unsigned)page < (unsigned)a.n_pages;
  const int d = a.head_dim, per = d >> 4;                  // per: units of a head
  const size_t slot = (size_t)(pos & ((1 << a.page_shift) - 1)) * d;
  const size_t head_step = (size_t)d << a.page_shift;
  const size_t page_at = ((size_t)a.layer * a.n_pages + (placed ? page : 0)) * a.n_kv_heads * head_step + slot;
  const float* turn = a.rotary ? a.rotary + (size_t)pos * a.dims : nullptr;
  const int nq = a.q ? a.n_heads * per : 0, nk = a.n_kv_heads * per;
  for (int w = threadIdx.x; w < nq + 2 * nk; w += kAppendThreads) {
    const int z = w < nq ? w : w < nq + nk ? w - nq : w - nq - nk;
    const int h = z / per, u = z % per;
    const uint16_t* row = w < nq ? a.q + (size_t)t * a.ld_q : w < nq + nk ? a.k + (size_t)t * a.ld_k : a.v + (size_t)t * a.ld_v;
    int i, j;
    chunks_of(u, a.dims, a.pairs, i, j);
    float x[8], y[8];
    load8(row + (size_t)h * d + i, x);
    load8(row + (size_t)h * d + j, y);
    if (w < nq + nk && turn && u < a.dims >> 4) turn_unit(x, y, turn, u, a.dims, a.pairs, 1.0f);
    if (w < nq) {
      put8<false>(a.q_out, (size_t)t * a.ld_q_out + (size_t)h * d + i, x, 1.0f);
      put8<false>(a.q_out, (size_t)t * a.ld_q_out + (size_t)h * d + j, y, 1.0f);
    } else if (placed) {
      const bool key = w < nq + nk;
      void* base = key ? a.k_cache : a.v_cache;
      const float scale = FP8 ? (key ? a.k_scale : a.v_scale)[(size_t)a.layer * a.n_kv_heads + h] : 1.0f;
      const size_t to = page_at + h * head_step;
      put8<FP8>(base, to + i, x, scale);
      put8<FP8>(base, to + j, y, scale);
    }
  }
}

// The same to a cache of blocks.  A block of a head's keys or values is one wavefront's work, from the largest of its values to its codes: it
// holds all of them in registers, or, where the call has few tokens for the block, several heads of it.  One workgroup per row turns the row's queries
// and takes its share of the heads of the block that the row is in, so that nothing has to be counted beforehand and a block's wavefronts are
// on different compute units.  Four prompts of about 1024 tokens (32 query, 8 key / value heads of 128): 93 MB in 21.5 us, 4.3 TB/s; 256 single tokens
// as long as a launch.
template <int D>
__global__ __launch_bounds__(kAppendThreads) void k_append_blocks(AppendArgs a) {
  constexpr int kUnits = D / 16, kRowsPass = 64 / kUnits, kPasses = MES_KV_BLOCK / kRowsPass;
  const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const Place at = place_of(a, t);
  const int pos = at.pos;
  const bool real = pos >= 0 && pos < a.capacity;
  const float* turns = a.rotary;
  if (a.q) append_queries(a, t, turns + (size_t)max(pos, 0) * a.dims, real);
  if (!real) return;
  const int page = a.page_table[(size_t)at.seq * a.table_pages + (pos >> a.page_shift)];
  if ((unsigned)page >= (unsigned)a.n_pages) return;
  const BlockRows in_call = block_rows(at, t, MES_KV_BLOCK);
  const int begin = in_call.begin, from = in_call.from, rows = in_call.rows, row0 = in_call.row0;
  const int older = from - begin, slot = begin & ((1 << a.page_shift) - 1);
  // lanes of a (head, keys or values), and how many of these a wavefront does at a time
  int lanes = kUnits;
  while (lanes < 64 && lanes < kUnits * rows) lanes <<= 1;
  const int together = 64 / lanes, l = lane & (lanes - 1), u = l % kUnits, r0 = l / kUnits, tasks = 2 * a.n_kv_heads;
  int i, j;
  chunks_of(u, a.dims, a.pairs, i, j);
  const bool turning = turns && u < a.dims >> 4;
  for (int group = wave * rows + (pos - from); group * together < tasks; group += kAppendThreads / 64 * rows) {
    const int task = group * together + lane / lanes;
    const bool mine = task < tasks, key = task < a.n_kv_heads;
    const int h = key ? task : task - a.n_kv_heads;
    float x[kPasses][8], y[kPasses][8], top = 0.0f;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int r = r0 + p * kRowsPass;
      if (!mine || r >= rows) continue;
      const uint16_t* row = (key ? a.k + (size_t)(row0 + r) * a.ld_k : a.v + (size_t)(row0 + r) * a.ld_v) + (size_t)h * D;
      load8(row + i, x[p]);
      load8(row + j, y[p]);
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int r = r0 + p * kRowsPass;
      if (!mine || r >= rows) continue;
      if (key && turning) turn_unit(x[p], y[p], turns + (size_t)(from + r) * a.dims, u, a.dims, a.pairs, 1.0f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float s = fabsf(x[p][e]), w = fabsf(y[p][e]);
        top = fmaxf(top, s <= 3.402823466e38f ? s : 0.0f);   // what is not finite does not count
        top = fmaxf(top, w <= 3.402823466e38f ? w : 0.0f);
      }
    }
    for (int m = 1; m < lanes; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
    if (!mine) continue;
    uint8_t* exponents = key ? a.k_exponent : a.v_exponent;
    uint8_t* codes = static_cast<uint8_t*>(key ? a.k_cache : a.v_cache) + ((((size_t)a.layer * a.n_pages + page) * a.n_kv_heads + h) << a.page_shift) * D;
    const size_t block = block_at(page, h, a.n_kv_heads, a.page_shift, slot);
    // the least with top <= 448 2^e, 448 = 1.75 2^8: 8 below top's own exponent, 7 where its mantissa is above 1.75
    int exponent = max((int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8, MES_KV_LEAST_EXPONENT);
    if (older) {
      const int was = exponent_of(exponents[block]);
      if (exponent > was) {                                  // seldom: a sequence's scale is found by its first tokens
        const float by = ldexpf(1.0f, was - exponent);
        for (int w = l; w < older * (D / 8); w += lanes) {
          uint2* p = reinterpret_cast<uint2*>(codes + (size_t)slot * D + w * 8);
          const uint2 c = *p;
          *p = make_uint2(scaled4(c.x, by), scaled4(c.y, by));
        }
      } else exponent = was;
    }
    if (l == 0) exponents[block] = (uint8_t)exponent;
    const float by = power_of(254 - exponent), limit = exponent == MES_KV_MOST_EXPONENT ? 240.0f : 448.0f;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int r = r0 + p * kRowsPass;
      if (r >= rows) continue;
      uint8_t* row = codes + (size_t)(slot + older + r) * D;
      *reinterpret_cast<uint2*>(row + i) = codes8(x[p], by, limit);
      *reinterpret_cast<uint2*>(row + j) = codes8(y[p], by, limit);
    }
  }
}

// Reading back: a thread 8 dimensions of a token, so that the stores of a wavefront are whole lines.  Workgroups take kReadRows rows; keys and
// values of a head are read in the order of the page, kReadBatch units of a thread on their way before the first is written.
// 64 contexts, 68 thousand tokens of 8 heads of 128: 407 MB in 91 us, 4.5 TB/s (4.88 is what a copy of 2 GiB reaches); workgroups of 16 and 32 rows, whose
// threads do more one after the other: 93 and 106.
constexpr int kReadThreads = 256, kReadRows = 8, kReadBatch = 8;

template <int DTYPE>
struct Codes8 {                                            // 8 dimensions as the cache holds them
  std::conditional_t<DTYPE == MES_KV_BF16, uint4, uint2> w;
  __device__ __forceinline__ void load(const void* base, size_t element) {
    w = *reinterpret_cast<const decltype(w)*>(static_cast<const char*>(base) + element * (DTYPE == MES_KV_BF16 ? 2 : 1));
  }
  __device__ __forceinline__ void store(uint16_t* to, float scale) const {
    uint4 v;
    if constexpr (DTYPE == MES_KV_BF16) {
      v = w;
    } else if constexpr (DTYPE == MES_KV_E4M3_BLOCKS) {
      v = make_uint4(widen2<false>(w.x, scale), widen2<true>(w.x, scale), widen2<false>(w.y, scale), widen2<true>(w.y, scale));
    } else {
      v = make_uint4(pack_bf16(code_at<0>(w.x) * scale, code_at<1>(w.x) * scale), pack_bf16(code_at<2>(w.x) * scale, code_at<3>(w.x) * scale),
                     pack_bf16(code_at<0>(w.y) * scale, code_at<1>(w.y) * scale), pack_bf16(code_at<2>(w.y) * scale, code_at<3>(w.y) * scale));
    }
    *reinterpret_cast<uint4*>(to) = v;
  }
};

template <int DTYPE, int D>
__global__ __launch_bounds__(kReadThreads) void k_read(ReadArgs a) {
  constexpr int kChunks = D / 8;
  __shared__ int pages[kReadRows], slots[kReadRows];       // page -1: absent, -2: no row of a sequence
  const int t0 = blockIdx.x * kReadRows;
  if (threadIdx.x < 64) {
    int seq = a.q_offsets ? sequence_of(a.q_offsets, a.n_seqs, t0) : t0;
    const int t = t0 + threadIdx.x;
    int page = -2, slot = 0;
    if (threadIdx.x < kReadRows && t < a.T) {
      if (a.q_offsets)
        while (seq < a.n_seqs && a.q_offsets[seq + 1] <= t) ++seq;
      else seq = t;
      const Place at = place_in(a, t, seq);
      if (at.seq >= 0) {
        page = -1;
        if (at.pos >= 0 && at.pos < a.capacity) {
          const int p = a.page_table[(size_t)at.seq * a.table_pages + (at.pos >> a.page_shift)];
          if ((unsigned)p < (unsigned)a.n_pages) page = p;
          slot = at.pos & ((1 << a.page_shift) - 1);
        }
      }
    }
    if (threadIdx.x < kReadRows) {
      pages[threadIdx.x] = page;
      slots[threadIdx.x] = slot;
    }
  }
  __syncthreads();
  const int half = a.n_kv_heads * kReadRows * kChunks;
  for (int w0 = threadIdx.x; w0 < 2 * half; w0 += kReadBatch * kReadThreads) {
    Codes8<DTYPE> codes[kReadBatch];
    float scale[kReadBatch];
    uint16_t* out[kReadBatch];
#pragma unroll
    for (int b = 0; b < kReadBatch; ++b) {
      const int w = w0 + b * kReadThreads;
      const bool key = w < half;
      const int z = key ? w : w - half, c = z % kChunks, r = z / kChunks % kReadRows, h = z / (kChunks * kReadRows);
      out[b] = key ? a.k : a.v;
      scale[b] = 1.0f;
      codes[b] = {};
      const int page = w < 2 * half ? pages[r] : -2, slot = slots[r];
      if (page == -2 && !(a.fresh && w < 2 * half && t0 + r < a.T)) out[b] = nullptr;
      if (!out[b]) continue;
      out[b] += (size_t)(t0 + r) * (key ? a.ld_k : a.ld_v) + (size_t)h * D + c * 8;
      if (page < 0) continue;                              // 0
      if constexpr (DTYPE == MES_KV_E4M3) scale[b] = (key ? a.k_scale : a.v_scale)[h];
      if constexpr (DTYPE == MES_KV_E4M3_BLOCKS) scale[b] = power_of(exponent_of((key ? a.k_exponent : a.v_exponent)[block_at(page, h, a.n_kv_heads, a.page_shift, slot)]));
      codes[b].load(key ? a.k_cache : a.v_cache, (((((size_t)page * a.n_kv_heads + h) << a.page_shift) + slot) * D) + c * 8);
    }
#pragma unroll
    for (int b = 0; b < kReadBatch; ++b)
      if (out[b]) codes[b].store(out[b], scale[b]);
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
  uint8_t *k_exponent, *v_exponent;    // nullptr: the cache has none
  size_t page_bytes, layer_bytes;
  int n_pages, page_exponents;
  int n_layers, parts;                 // parts: workgroups per page of a layer
  int32_t src[kCopyPairs], dst[kCopyPairs];
};

__global__ __launch_bounds__(kCopyThreads) void k_copy_pages(CopyArgs a) {
  const int part = blockIdx.x % a.parts, layer = (blockIdx.x / a.parts) % a.n_layers, pair = blockIdx.x / a.parts / a.n_layers;
  char* base = (blockIdx.y ? a.v : a.k) + layer * a.layer_bytes;
  const size_t at = (size_t)part * kCopyBytes + threadIdx.x * 16;
  if (part == 0 && a.k_exponent) {
    uint8_t* of = (blockIdx.y ? a.v_exponent : a.k_exponent) + (size_t)layer * a.n_pages * a.page_exponents;
    for (int x = threadIdx.x; x < a.page_exponents; x += kCopyThreads) of[(size_t)a.dst[pair] * a.page_exponents + x] = of[(size_t)a.src[pair] * a.page_exponents + x];
  }
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

hipError_t launch_append(const AppendArgs& a, int dtype, hipStream_t s) {
  const int T = a.T;
  if (dtype == MES_KV_BF16) k_append<false><<<T, kAppendThreads, 0, s>>>(a);
  else if (dtype == MES_KV_E4M3) k_append<true><<<T, kAppendThreads, 0, s>>>(a);
  else if (a.head_dim == 128) k_append_blocks<128><<<T, kAppendThreads, 0, s>>>(a);
  else k_append_blocks<64><<<T, kAppendThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_read(const ReadArgs& a, int dtype, hipStream_t s) {
  const unsigned grid = (unsigned)((a.T + kReadRows - 1) / kReadRows);
  auto go = [&](auto type) {
    constexpr int DTYPE = decltype(type)::value;
    if (a.head_dim == 128) k_read<DTYPE, 128><<<grid, kReadThreads, 0, s>>>(a);
    else k_read<DTYPE, 64><<<grid, kReadThreads, 0, s>>>(a);
  };
  if (dtype == MES_KV_BF16) go(std::integral_constant<int, MES_KV_BF16>{});
  else if (dtype == MES_KV_E4M3) go(std::integral_constant<int, MES_KV_E4M3>{});
  else go(std::integral_constant<int, MES_KV_E4M3_BLOCKS>{});
  return hipGetLastError();
}

hipError_t launch_copy_pages(const mes_kv& kv, const int32_t* src, const int32_t* dst, int n, hipStream_t s) {
  CopyArgs a;
  a.k = static_cast<char*>(kv.k);
  a.v = static_cast<char*>(kv.v);
  a.page_bytes = (size_t)kv.n_kv_heads * kv.page_tokens * kv.head_dim * (kv.dtype == MES_KV_BF16 ? 2 : 1);
  a.k_exponent = kv.dtype == MES_KV_E4M3_BLOCKS ? kv.k_exponent : nullptr;
  a.v_exponent = kv.dtype == MES_KV_E4M3_BLOCKS ? kv.v_exponent : nullptr;
  a.n_pages = kv.n_pages;
  a.page_exponents = kv.n_kv_heads * kv.page_tokens / MES_KV_BLOCK;
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
