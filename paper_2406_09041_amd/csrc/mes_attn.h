// Declarations shared by the attention and cache translation units (not part of the ABI).
#pragma once

#include <algorithm>

#include "mes_internal.h"

namespace mes {

// Page pairs of one copy launch: its arguments stay below 4 KiB.
constexpr int kCopyPairs = 480;

// The power of two that a block's exponent stands for, and the exponent inside the bytes that are written.
constexpr int kBlockShift = 4;
static_assert(1 << kBlockShift == MES_KV_BLOCK, "tokens of a block");
__device__ __forceinline__ int exponent_of(int byte) { return min(max(byte, MES_KV_LEAST_EXPONENT), MES_KV_MOST_EXPONENT); }
__device__ __forceinline__ float power_of(int exponent) { return __uint_as_float((uint32_t)exponent << 23); }
// a block's exponent: page, head and slot of a layer
__device__ __forceinline__ size_t block_at(int page, int head, int n_kv_heads, int page_shift, int slot) {
  return ((((size_t)page * n_kv_heads + head) << page_shift) + slot) >> kBlockShift;
}

// ---- implemented in mes_cache.hip --------------------------------------------------------------
struct AppendArgs {
  const uint16_t *q, *k, *v;
  const float* rotary;
  uint16_t* q_out;
  void *k_cache, *v_cache;
  const float *k_scale, *v_scale;      // e4m3
  uint8_t *k_exponent, *v_exponent;    // blocks; of the layer
  const int32_t *q_offsets, *kv_len, *page_table;
  int T, layer, n_pages, page_shift, n_heads, n_kv_heads, head_dim, n_seqs, table_pages, capacity;
  int ld_q, ld_k, ld_v, ld_q_out;
  int dims;                            // that are turned
  bool pairs;                          // of neighbours
  bool fresh;                          // rows of q_out that get nothing are set to 0
};
hipError_t launch_append(const AppendArgs& a, int dtype, hipStream_t s);
struct ReadArgs {
  const void *k_cache, *v_cache;       // the cache's layer
  const float *k_scale, *v_scale;      // of the layer, e4m3
  const uint8_t *k_exponent, *v_exponent;
  uint16_t *k, *v;                     // nullptr: not wanted
  const int32_t *q_offsets, *kv_len, *page_table;
  int T, n_pages, page_shift, n_kv_heads, head_dim, n_seqs, table_pages, capacity, ld_k, ld_v;
  bool fresh;
};
hipError_t launch_read(const ReadArgs& a, int dtype, hipStream_t s);
hipError_t launch_copy_pages(const mes_kv& kv, const int32_t* src, const int32_t* dst, int n, hipStream_t s);

// ---- implemented in mes_rotary.hip --------------------------------------------------------------
constexpr int kMostTurned = 512;       // dimensions
struct TableArgs {
  float* table;
  int64_t n_positions;
  int dims;
  double magnitude, frequency[kMostTurned / 2];
};
hipError_t launch_rotary_table(const TableArgs& a, hipStream_t s);
struct RotaryArgs {
  const void *q, *k;
  void *q_out, *k_out;
  const int32_t* positions;
  const float* table;
  int T, n_heads, n_kv_heads, head_dim, ld_q, ld_k, ld_q_out, ld_k_out, n_positions, dims;
  float sign;
  bool pairs, fresh;
};
hipError_t launch_rotary(const RotaryArgs& a, bool fp32, hipStream_t s);

// ---- implemented in mes_attn_prompt.hip ---------------------------------------------------------
struct PromptArgs {
  const uint16_t *q, *k, *v;           // k, v: packed rows, or the cache's layer
  uint16_t* out;
  const float *k_scale, *v_scale;      // of the layer, e4m3 caches only
  const uint8_t *k_exponent, *v_exponent;   // of the layer, blocks only
  const int32_t *q_offsets, *kv_len, *page_table;   // kv_len, page_table: cache only
  int T, n_seqs, n_heads, n_kv_heads, head_dim, n_pages, page_shift, table_pages, capacity;
  int ld_q, ld_k, ld_v, ld_out;
  float scale;
  void* ws;                            // nullptr: no item is cut
};
enum { KV_PACKED = 0, KV_PAGED = 1, KV_PAGED_E4M3 = 2, KV_PAGED_BLOCKS = 3 };
size_t attn_prompt_workspace_bytes(int T, int n_seqs, int n_heads, int n_kv_heads, int head_dim);
hipError_t launch_attn_prompt(const PromptArgs& a, int source, hipStream_t s);

// ---- implemented in mes_attn_decode.hip ---------------------------------------------------------
struct DecodeArgs {
  const uint16_t* q;
  const void *k, *v;                   // the cache's layer
  uint16_t* out;
  const float *k_scale, *v_scale;
  const uint8_t *k_exponent, *v_exponent;
  const int32_t *kv_len, *page_table;
  void* ws;
  int n_seqs, n_heads, n_kv_heads, head_dim, n_pages, page_shift, table_pages, capacity, ld_q, ld_out;
  float scale;
  int n_groups;                        // of sequences that share a prefix (two of them at least): rows first .. behind
  int32_t first[MES_MAX_EXPERTS], behind[MES_MAX_EXPERTS], prefix[MES_MAX_EXPERTS];
};
// Of the first `prefix` tokens, which an expert's sequences share, those that one sequence's pages give for all of them.  Over blocks whole blocks: the one
// that the prefix ends in also holds tokens of the sequence's own, which have a part in its exponent and so in the prefix's codes.
__host__ __device__ constexpr int shared_tokens(bool blocks, int prefix) { return blocks ? prefix & -MES_KV_BLOCK : prefix; }
// Work of a decode call is numbered in 32 bits, in costs: of a sequence and key / value head there are at most kMostCosts (u + 2), u = page table's tokens / 128
// (mes_attn_decode.hip has the proof), and calls that could have 2^32 are refused.
constexpr int64_t kMostCosts = 12;
inline bool decode_fits(int n_seqs, int n_kv_heads, int capacity) { return kMostCosts * n_seqs * n_kv_heads * (capacity / 128 + 2) <= (int64_t)1 << 32; }
size_t attn_decode_workspace_bytes(int n_seqs, int n_heads, int n_kv_heads, int head_dim);
hipError_t launch_attn_decode(const DecodeArgs& a, int source, hipStream_t s);

}  // namespace mes
