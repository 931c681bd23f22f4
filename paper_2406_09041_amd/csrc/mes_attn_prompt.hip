// Causal attention over packed prompts, and over new tokens behind a paged cache.  Bound by the matrix cores (and the
// exponentials between their products); the mathematics, per query row n with scores s_j = scale * <q, k_j>:
//   m = max s_j (kept within kSlack of it), p_j = 2^(s_j log2e - m), l = sum p_j, o = sum p_j v_j / l
// in one pass over the keys, 64 at a time, nothing of the scores in memory.
//
// A workgroup takes kRows = 128 query rows of one head, a wavefront 32 of them.  The scores are formed transposed,
// S^T = K Q^T: in the result of v_mfma_f32_32x32x16_bf16 a lane then holds ONE query row (column lane & 31) and 16 of 32
// keys, so that maxima, sums and rescaling need no exchange but one with lane ^ 32, and its registers, rounded to bf16, ARE the
// operand P^T of the second product O^T = V^T P^T: keys 4 h + (0..3) and 8 + 4 h + (0..3) of every 16 for half h
// of the wavefront.  V's operand for these keys is read from LDS with the transposing read (ds_read_b64_tr_b16), in the
// order of the keys that P has.  O^T keeps query rows on lanes as well.
//
// Keys and values stand in LDS as rows of head_dim, two tiles of 64 in turn (one arrives while the other is multiplied).
// Rows are 256 (128) bytes, so that all rows would start in the same bank: the 16-byte pieces of row r are XORed with
// swizzle(r), which spreads both the 32 rows that a K operand reads at one piece and the 4 rows x 64 bytes of a
// transposing read over all banks.  The copy into LDS writes 16 bytes per lane in order, so the permutation is
// applied to the address that a lane fetches.
#include "mes_attn_common.h"

namespace mes {
namespace {

constexpr int kRows = 128, kTile = 64, kThreads = 256;

template <int D>
__device__ __forceinline__ int swizzle(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

// What an absent token (behind the sequence's end, or on a page that does not exist) is read from: its value row must
// not be able to turn a weight of 0 into NaN.
__device__ const u32x4 g_zeros[16] = {};

__device__ __forceinline__ void copy_to_lds(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(to) : "memory", "m0");
}

// The part of the call a workgroup works on: query rows [first, first + rows) of the sequence's `behind` rows
struct Item {
  int seq, row0, rows, tile, before;   // sequence; its first row in the call; its rows; tile of kRows of them; tokens before row 0
};

// Item j of the call.  Up to 64 sequences: items in order of the keys they see, most first (in units of kRows), so that no long
// one starts last; lane s counts for sequence s.  More: tile t of sequence s has number floor(o[s] / kRows) + s + t, which leaves gaps
// (no item) but needs no sum over the sequences before it; the last first, as they see most of their sequence.
template <int SRC>
__device__ bool find_item(const PromptArgs& a, int j, int slots, Item& it) {
  const int lane = threadIdx.x & 63;
  auto rows_of = [&](int s, int& lo) {
    lo = min(max(a.q_offsets[s], 0), a.T);
    return max(min(a.q_offsets[s + 1], a.T) - lo, 0);
  };
  if (a.n_seqs <= 64) {
    int lo = 0, n = 0, before = 0;
    if (lane < a.n_seqs) {
      n = rows_of(lane, lo);
      if (SRC != KV_PACKED) before = max(a.kv_len[lane], 0) - n;
    }
    const int tiles = (n + kRows - 1) / kRows, base = max(before, 0) / kRows;
    if (j >= wave_sum(tiles)) return false;
    // the level L with C(L + 1) <= j < C(L), C(L) = number of tiles with base + t >= L
    auto count = [&](int level) { return wave_sum(min(max(base + tiles - max(level, base), 0), tiles)); };
    int low = 0, high = wave_max(base + tiles);           // C(low) > j >= C(high) = 0
    while (high - low > 1) {
      const int mid = low + (high - low) / 2;
      if (count(mid) > j) low = mid; else high = mid;
    }
    const int rank = j - count(low + 1);
    const bool mine = base <= low && low < base + tiles;
    const uint64_t who = __ballot(mine);
    const bool chosen = mine && __popcll(who & ((1ull << lane) - 1)) == rank;
    const int s = __builtin_ctzll(__ballot(chosen));
    it.seq = s;
    it.row0 = __shfl(lo, s);
    it.rows = __shfl(n, s);
    it.before = __shfl(before, s);
    it.tile = low - __shfl(base, s);
    return true;
  }
  j = slots - 1 - j;
  int lo = 0, hi = a.n_seqs - 1;                           // last s with floor(o[s] / kRows) + s <= j
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (max(a.q_offsets[mid], 0) / kRows + mid <= j) lo = mid; else hi = mid - 1;
  }
  it.seq = lo;
  it.rows = rows_of(lo, it.row0);
  it.tile = j - max(a.q_offsets[lo], 0) / kRows - lo;
  it.before = SRC != KV_PACKED ? max(a.kv_len[lo], 0) - it.rows : 0;
  return it.tile >= 0 && it.tile < (it.rows + kRows - 1) / kRows;
}

template <int D, int SRC>
__global__ __launch_bounds__(kThreads, 2) void k_attn_prompt(PromptArgs a, int slots) {
  constexpr int kPieces = D / 8, kRowBytes = D * 2, kTileBytes = kTile * kRowBytes;   // pieces of 16 bytes
  constexpr int KS = D / 16, DT = D / 32;
  constexpr int kCopies = kTileBytes / (kThreads * 16);                              // copies of 16 bytes per lane and tile
  __shared__ __align__(16) char lds[2][2][kTileBytes];                               // [buffer][keys, values]
  __shared__ int lds_there[2][4];                                                    // whether 16 keys of a tile have a page
  __shared__ int lds_again;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int col = lane & 31, half = lane >> 5;

  Item it;
  if (!find_item<SRC>(a, blockIdx.x / a.n_heads, slots, it)) return;
  it.seq = uniform(it.seq); it.row0 = uniform(it.row0); it.rows = uniform(it.rows); it.tile = uniform(it.tile); it.before = uniform(it.before);
  // consecutive workgroups go to the XCDs in turn: the heads that share keys and values come n_kv_heads apart, which puts them
  // on one XCD (8, 16, 40 ... key / value heads), whose L2 then fetches them once
  const int hx = blockIdx.x % a.n_heads, kvh = hx % a.n_kv_heads, head = kvh * (a.n_heads / a.n_kv_heads) + hx / a.n_kv_heads;

  const int row_first = it.tile * kRows, row_count = min(kRows, it.rows - row_first);
  // keys [0, kv_end) are seen by some row of the workgroup
  const int capacity = SRC == KV_PACKED ? 0x7fffffff : a.capacity;
  const int kv_end = min(it.before + row_first + row_count, capacity);
  const int n_tiles = kv_end > 0 ? (kv_end + kTile - 1) / kTile : 0;
  const int my_row = row_first + 32 * wave + col;                  // of the sequence's rows
  const int pos = it.before + my_row;                              // sees keys <= pos
  const int pos_low = it.before + row_first + 32 * wave, pos_high = min(pos_low + 31, it.before + it.rows - 1);

  // Q^T operand: lane (col, half) holds dimensions 16 ks + 8 half + (0..7) of its row
  bf16x8 q[KS];
  {
    const uint16_t* src = a.q + (size_t)(it.row0 + min(my_row, it.rows - 1)) * a.ld_q + (size_t)head * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) q[ks] = *reinterpret_cast<const bf16x8*>(src + 16 * ks);
  }
  const float scale = a.scale * kLog2e * (SRC == KV_PAGED_E4M3 ? a.k_scale[kvh] : 1.0f);

  // ---- staging: wavefront w brings keys 16 w .. 16 w + 15 of every tile
  const int32_t* table = SRC == KV_PACKED ? nullptr : a.page_table + (size_t)it.seq * a.table_pages;
  int page_next = 0;                                               // page of this wavefront's 16 keys of the tile requested next
  auto look_up = [&](int tile) {
    if constexpr (SRC != KV_PACKED) {
      const int token = tile * kTile + 16 * wave;
      page_next = token < kv_end ? table[token >> a.page_shift] : -1;
    }
  };
  u32x4 raw[2][2];                                                 // e4m3: a tile's codes on their way
  auto request = [&](int tile, int buffer) {
    const int token0 = tile * kTile + 16 * wave;
    if constexpr (SRC == KV_PACKED || SRC == KV_PAGED) {
      size_t base_k, base_v, step_k, step_v;
      bool there = true;
      if constexpr (SRC == KV_PACKED) {
        base_k = ((size_t)it.row0 + token0) * a.ld_k + (size_t)kvh * D;
        base_v = ((size_t)it.row0 + token0) * a.ld_v + (size_t)kvh * D;
        step_k = a.ld_k;
        step_v = a.ld_v;
      } else {
        const int page = uniform(page_next);
        there = (unsigned)page < (unsigned)a.n_pages;
        base_k = base_v = ((((size_t)(there ? page : 0) * a.n_kv_heads + kvh) << a.page_shift) + (token0 & ((1 << a.page_shift) - 1))) * D;
        step_k = step_v = D;
        if (lane == 0) lds_there[buffer][wave] = there;
      }
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const int r = i * (64 / kPieces) + lane / kPieces;          // of the wavefront's 16 rows
        const int piece = (lane % kPieces) ^ swizzle<D>(16 * wave + r);
        const bool real = there && token0 + r < kv_end;
        const void* from_k = real ? (const void*)(a.k + base_k + r * step_k + piece * 8) : (const void*)&g_zeros[piece];
        const void* from_v = real ? (const void*)(a.v + base_v + r * step_v + piece * 8) : (const void*)&g_zeros[piece];
        const uint32_t at = (16 * wave + i * (64 / kPieces)) * kRowBytes;
        copy_to_lds(from_k, (uint32_t)(uintptr_t)&lds[buffer][0][at]);
        copy_to_lds(from_v, (uint32_t)(uintptr_t)&lds[buffer][1][at]);
      }
    } else {
      // four lanes per key, head_dim / 4 codes each
      const int page = uniform(page_next), r = lane >> 2, part = lane & 3;
      const bool there = (unsigned)page < (unsigned)a.n_pages;
      if (lane == 0) lds_there[buffer][wave] = there;
      const size_t at = ((((size_t)(there ? page : 0) * a.n_kv_heads + kvh) << a.page_shift) + (token0 & ((1 << a.page_shift) - 1)) + r) * D + part * (D / 4);
      const bool real = there && token0 + r < kv_end;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        raw[0][i] = real ? *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(a.k) + at + 16 * i) : u32x4{0, 0, 0, 0};
        raw[1][i] = real ? *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(a.v) + at + 16 * i) : u32x4{0, 0, 0, 0};
      }
    }
  };
  auto deposit = [&](int buffer) {                                   // e4m3: codes -> bf16 rows in LDS
    if constexpr (SRC == KV_PAGED_E4M3) {
      const int r = 16 * wave + (lane >> 2), part = lane & 3;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const u32x2 x = widen4(raw[kv][i / 2][2 * (i % 2)]), y = widen4(raw[kv][i / 2][2 * (i % 2) + 1]);
          *reinterpret_cast<u32x4*>(&lds[buffer][kv][r * kRowBytes + (((part * (D / 32) + i) ^ swizzle<D>(r)) * 16)]) = u32x4{x[0], x[1], y[0], y[1]};
        }
    }
  };

  f32x16 acc[DT];
  float m, l;
  // A value of a key that a row does not see can still be infinite or NaN, and a weight of 0 times it is NaN: seen at the
  // end, and then all is done once more with the tiles that hold keys not everybody sees taken key by key.
  for (int careful = 0; careful < 2; ++careful) {
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[dt][i] = 0.0f;
    __syncthreads();                                                 // the buffers are free
    if (threadIdx.x == 0) lds_again = 0;
    if (n_tiles > 0) {
      look_up(0);
      request(0, 0);
      look_up(1);
      deposit(0);
    }
    for (int kt = 0; kt < n_tiles; ++kt) {
      const int buffer = kt & 1;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();                                               // tile kt is there, and nobody reads the other buffer any more
      if (kt + 1 < n_tiles) {
        request(kt + 1, buffer ^ 1);
        look_up(kt + 2);
      }
      const int key0 = kt * kTile;
      if (key0 <= pos_high) {
        const char* lk = lds[buffer][0];
        const char* lv = lds[buffer][1];
        int there = 15;
        if constexpr (SRC != KV_PACKED)
          there = uniform(lds_there[buffer][0] | lds_there[buffer][1] << 1 | lds_there[buffer][2] << 2 | lds_there[buffer][3] << 3);
        const bool masked = key0 + kTile - 1 > pos_low || key0 + kTile > kv_end || there != 15;
        if (!(masked && careful)) {
          f32x16 s[2];
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[tt][i] = 0.0f;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
              const int r = 32 * tt + col;
              const bf16x8 k = *reinterpret_cast<const bf16x8*>(lk + r * kRowBytes + (((2 * ks + half) ^ swizzle<D>(r)) * 16));
              s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[ks], s[tt], 0, 0, 0);
            }
          if (masked) {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int r = 32 * tt + 8 * (i / 4) + 4 * half + i % 4;
                if (key0 + r > pos || key0 + r >= kv_end || !((there >> (r >> 4)) & 1)) s[tt][i] = -INFINITY;
              }
          }
          float top = -INFINITY;
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[tt][i]);
          if (__any(top * scale > m + kSlack)) {
            top = fmaxf(top, other_half(top)) * scale;
            const float raised = fmaxf(m, top);
            const float to = raised == -INFINITY ? 0.0f : raised;
            const float shrink = exp2_fast(m - to);
            l *= shrink;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int i = 0; i < 16; ++i) acc[dt][i] *= shrink;
            m = raised;
          }
          const float from = m == -INFINITY ? 0.0f : m;
          u32x4 p[4];                                                // 16 keys each
#pragma unroll
          for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int tt = st / 2, e = 8 * (st % 2) + 2 * i;
              p[st][i] = pack2(exp2_fast(s[tt][e] * scale - from), exp2_fast(s[tt][e + 1] * scale - from));
              l = add_pair(p[st][i], l);                             // the sum of what is multiplied with V
            }
          // V^T operands: lanes of 16 read 4 keys x 16 dimensions, 8 bytes each, and get a dimension's 4 keys
#pragma unroll
          for (int st = 0; st < 4; ++st) {
            const int r = 16 * st + 4 * half + ((lane & 15) >> 2);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
              const int piece = 4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
              typedef __attribute__((address_space(3))) i16x4* lds_ptr;
              const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lv + r * kRowBytes + ((piece ^ swizzle<D>(r)) * 16) + 8 * (lane & 1)));
              const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lv + (r + 8) * kRowBytes + ((piece ^ swizzle<D>(r + 8)) * 16) + 8 * (lane & 1)));
              struct { i16x4 lo, hi; } v = {lo, hi};
              acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p[st]), acc[dt], 0, 0, 0);
            }
          }
        } else {
          for (int r = 0; r < min(kTile, kv_end - key0); ++r) {      // key by key, rows that do not see it untouched
            float dot = 0.0f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
              const bf16x8 k = *reinterpret_cast<const bf16x8*>(lk + r * kRowBytes + (((2 * ks + half) ^ swizzle<D>(r)) * 16));
#pragma unroll
              for (int e = 0; e < 8; ++e) dot = fmaf((float)k[e], (float)q[ks][e], dot);
            }
            dot = (dot + other_half(dot)) * scale;
            const bool seen = key0 + r <= pos && ((there >> (r >> 4)) & 1);
            const float raised = seen && dot > m + kSlack ? dot : m;
            const float shrink = raised == m ? 1.0f : exp2_fast(m - raised);
            const float w = bf16_at(pack2(exp2_fast(dot - (raised == -INFINITY ? 0.0f : raised)), 0.0f), 0);
            m = raised;
            l = seen ? l * shrink + 0.5f * w : l;                    // the halves' sums are added at the end
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
              for (int i4 = 0; i4 < 4; ++i4) {
                const u32x2 v = *reinterpret_cast<const u32x2*>(lv + r * kRowBytes + (((4 * dt + i4) ^ swizzle<D>(r)) * 16) + 8 * half);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const float x = acc[dt][4 * i4 + i];
                  acc[dt][4 * i4 + i] = seen ? fmaf(w, bf16_at(v[i / 2], i % 2), x * shrink) : x;
                }
              }
          }
        }
      }
      deposit(buffer ^ 1);
    }
    if (careful) break;
    float test = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) test = fmaf(acc[dt][i], 0.0f, test);
    if (my_row < it.rows && test != test) lds_again = 1;
    __syncthreads();
    if (!uniform(lds_again)) break;
  }

  l += other_half(l);
  if (my_row >= it.rows) return;
  const float inv = l == 0.0f ? 0.0f : (SRC == KV_PAGED_E4M3 ? a.v_scale[kvh] : 1.0f) / l;
  uint16_t* dst = a.out + (size_t)(it.row0 + my_row) * a.ld_out + (size_t)head * D + 4 * half;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<u32x2*>(dst + 32 * dt + 8 * i) =
          u32x2{pack2(acc[dt][4 * i] * inv, acc[dt][4 * i + 1] * inv), pack2(acc[dt][4 * i + 2] * inv, acc[dt][4 * i + 3] * inv)};
}

template <int D>
hipError_t launch(const PromptArgs& a, int source, hipStream_t s) {
  // enough items for every way T rows can be shared out over the sequences
  const int64_t slots = (int64_t)a.T / kRows + a.n_seqs;
  if (slots * a.n_heads > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(slots * a.n_heads));
  if (source == KV_PACKED) k_attn_prompt<D, KV_PACKED><<<grid, kThreads, 0, s>>>(a, (int)slots);
  else if (source == KV_PAGED) k_attn_prompt<D, KV_PAGED><<<grid, kThreads, 0, s>>>(a, (int)slots);
  else k_attn_prompt<D, KV_PAGED_E4M3><<<grid, kThreads, 0, s>>>(a, (int)slots);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_prompt(const PromptArgs& a, int source, hipStream_t s) {
  return a.head_dim == 128 ? launch<128>(a, source, s) : launch<64>(a, source, s);
}

}  // namespace mes
