// Declarations shared by the attention and cache translation units (not part of the ABI).
#pragma once

#include <algorithm>

#include "mes_internal.h"

namespace mes {

// Page pairs of one copy launch: its arguments stay below 4 KiB.
constexpr int kCopyPairs = 480;

// ---- implemented in mes_cache.hip --------------------------------------------------------------
struct AppendArgs {
  const uint16_t *q, *k, *v;
  const float* rotary;
  uint16_t* q_out;
  void *k_cache, *v_cache;
  const float *k_scale, *v_scale;
  const int32_t *q_offsets, *kv_len, *page_table;
  int layer, n_pages, page_shift, n_heads, n_kv_heads, head_dim, n_seqs, table_pages, capacity;
  int ld_q, ld_k, ld_v, ld_q_out;
  bool fresh;                          // rows of q_out that get nothing are set to 0
};
hipError_t launch_append(const AppendArgs& a, int T, bool fp8, hipStream_t s);
hipError_t launch_copy_pages(const mes_kv& kv, const int32_t* src, const int32_t* dst, int n, hipStream_t s);

// ---- implemented in mes_attn_prompt.hip ---------------------------------------------------------
struct PromptArgs {
  const uint16_t *q, *k, *v;           // k, v: packed rows, or the cache's layer
  uint16_t* out;
  const float *k_scale, *v_scale;      // of the layer, e4m3 caches only
  const int32_t *q_offsets, *kv_len, *page_table;   // kv_len, page_table: cache only
  int T, n_seqs, n_heads, n_kv_heads, head_dim, n_pages, page_shift, table_pages, capacity;
  int ld_q, ld_k, ld_v, ld_out;
  float scale;
  void* ws;                            // nullptr: no item is cut
};
enum { KV_PACKED = 0, KV_PAGED = 1, KV_PAGED_E4M3 = 2 };
size_t attn_prompt_workspace_bytes(int T, int n_seqs, int n_heads, int n_kv_heads, int head_dim);
hipError_t launch_attn_prompt(const PromptArgs& a, int source, hipStream_t s);

// ---- implemented in mes_attn_decode.hip ---------------------------------------------------------
struct DecodeArgs {
  const uint16_t* q;
  const void *k, *v;                   // the cache's layer
  uint16_t* out;
  const float *k_scale, *v_scale;
  const int32_t *kv_len, *page_table;
  void* ws;
  int n_seqs, n_heads, n_kv_heads, head_dim, n_pages, page_shift, table_pages, capacity, ld_q, ld_out;
  float scale;
  int n_groups;                        // of sequences that share a prefix (two of them at least): rows first .. behind
  int32_t first[MES_MAX_EXPERTS], behind[MES_MAX_EXPERTS], prefix[MES_MAX_EXPERTS];
};
size_t attn_decode_workspace_bytes(int n_seqs, int n_heads, int n_kv_heads, int head_dim);
hipError_t launch_attn_decode(const DecodeArgs& a, bool fp8, hipStream_t s);

}  // namespace mes
