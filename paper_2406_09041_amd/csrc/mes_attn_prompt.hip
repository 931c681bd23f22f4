// Causal attention over packed prompts, and over new tokens behind a paged cache.  Bound by the matrix cores (and the
// exponentials between their products); the mathematics, per query row with scores s_j = scale * <q, k_j>:
//   m = max s_j (kept within kSlack of it), p_j = 2^(s_j log2e - m), l = sum p_j, o = sum p_j v_j / l
// in one pass over the keys, 64 at a time, nothing of the scores in memory (mes_attn_tiles.h).
//
// A workgroup is 4 wavefronts of 64 query rows: of up to 4 heads that share keys and values (all of them then see as many keys,
// and no wavefront waits for another), else of consecutive rows of one head.
#include "mes_attn_tiles.h"

namespace mes {
namespace {

// The part of the call a workgroup works on
struct Item {
  int seq, row0, rows, tile, before;   // sequence; its first row in the call; its rows; tile of R of them; tokens before row 0
};

// Item j of the call.  Up to 64 sequences: items in order of the keys they see, most first (in units of R rows), so that no long
// one starts last; lane s counts for sequence s.  More: tile t of sequence s has number floor(o[s] / R) + s + t, which leaves gaps
// (no item) but needs no sum over the sequences before it; the last first, as they see most of their sequence.
template <int SRC>
__device__ bool find_item(const PromptArgs& a, int R, int j, int slots, Item& it) {
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
    const int tiles = (n + R - 1) / R, base = max(before, 0) / R;
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
  int lo = 0, hi = a.n_seqs - 1;                           // last s with floor(o[s] / R) + s <= j
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (max(a.q_offsets[mid], 0) / R + mid <= j) lo = mid; else hi = mid - 1;
  }
  it.seq = lo;
  it.rows = rows_of(lo, it.row0);
  it.tile = j - max(a.q_offsets[lo], 0) / R - lo;
  it.before = SRC != KV_PACKED ? max(a.kv_len[lo], 0) - it.rows : 0;
  return it.tile >= 0 && it.tile < (it.rows + R - 1) / R;
}

// Every row once more, key by key and with no key that it does not see: the way out where a value that some rows do not see is infinite
// or NaN (a weight of 0 times it is NaN, also in the rows that must not notice).
template <int D, int SRC>
__device__ __forceinline__ void attend_by_key(TileRows<D>& w, Stage<D, SRC>& stage, int n_all, const int (&last)[NB], float scale) {
  constexpr int KS = D / 16, DT = D / 32;
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    w.m[b] = -INFINITY;
    w.l[b] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) w.acc[b][dt] = f32x16{};
  }
  stage.batch = -64;
  for (int t = 0; t < n_all; ++t) {
    barrier();                                                      // nobody reads the tiles of LDS any more
    stage.look_up(t);
    stage.request(t, 0);
    stage.deposit(t, 0);
    stage.request(t, 1);
    stage.deposit(t, 1);
    stage.arrive();
    barrier();
    const char* lk = stage.slot(t, 0);
    const char* lv = stage.slot(t, 1);
    const int there = stage.there(t);
    for (int r = 0; r < min(kTile, stage.to - t * kTile); ++r) {
      if (!((there >> (r >> 4)) & 1)) continue;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float dot = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const bf16x8 k = *reinterpret_cast<const bf16x8*>(lk + Row<D>::at(r) + (((2 * ks + half) ^ Row<D>::turn(r)) * 16));
#pragma unroll
          for (int e = 0; e < 8; ++e) dot = fmaf((float)k[e], (float)w.q[b][ks][e], dot);
        }
        dot = (dot + other_half(dot)) * scale;
        const bool seen = t * kTile + r <= last[b];
        const float raised = seen && dot > w.m[b] + kSlack ? dot : w.m[b];
        const float shrink = raised == w.m[b] ? 1.0f : exp2_fast(w.m[b] - raised);
        const float weight = bf16_at(pack2(exp2_fast(dot - (raised == -INFINITY ? 0.0f : raised)), 0.0f), 0);
        w.m[b] = raised;
        w.l[b] = seen ? w.l[b] * shrink + 0.5f * weight : w.l[b];   // the halves' sums are added at the end
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(lv + Row<D>::at(r) + (((4 * dt + i4) ^ Row<D>::turn(r)) * 16) + 8 * half);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x = w.acc[b][dt][4 * i4 + i];
              w.acc[b][dt][4 * i4 + i] = seen ? fmaf(weight, bf16_at(v[i / 2], i % 2), x * shrink) : x;
            }
          }
      }
    }
  }
}

// heads: heads of one workgroup (1, 2 or 4, a divisor of the heads per key / value head)
template <int D, int SRC>
__global__ __launch_bounds__(kTileThreads, 2) void k_attn_prompt(PromptArgs a, int slots, int heads) {
  constexpr int KS = D / 16, DT = D / 32;
  __shared__ __align__(16) TileLds<D> lds;
  __shared__ int lds_again;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int R = 4 * kWaveRows / heads, columns = a.n_heads / heads;  // rows of an item, workgroups of one item

  Item it;
  if (!find_item<SRC>(a, R, blockIdx.x / columns, slots, it)) return;
  it.seq = uniform(it.seq); it.row0 = uniform(it.row0); it.rows = uniform(it.rows); it.tile = uniform(it.tile); it.before = uniform(it.before);
  // consecutive workgroups go to the XCDs in turn: those that share keys and values come n_kv_heads apart, which puts them on
  // one XCD (8, 16, 40 ... key / value heads), whose L2 then fetches them once
  const int hx = blockIdx.x % columns, kvh = hx % a.n_kv_heads;
  const int head = kvh * (a.n_heads / a.n_kv_heads) + hx / a.n_kv_heads * heads + wave % heads;

  // keys [0, kv_end) are seen by some row of the workgroup
  const int row_first = it.tile * R, capacity = SRC == KV_PACKED ? 0x7fffffff : a.capacity;
  const int kv_end = min(it.before + min(row_first + R, it.rows), capacity);
  const int n_all = kv_end > 0 ? (kv_end + kTile - 1) / kTile : 0;
  const int wave_row = row_first + wave / heads * kWaveRows;         // the wavefront's first row
  const int high = min(it.before + min(wave_row + kWaveRows, it.rows), capacity);   // keys seen by its last row
  const int n = wave_row < it.rows && high > 0 ? (high + kTile - 1) / kTile : 0;
  int last[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) last[b] = it.before + wave_row + 32 * b + col;

  Stage<D, SRC> stage(lds);
  stage.kvh = kvh;
  stage.to = kv_end;
  if constexpr (SRC == KV_PACKED) {
    stage.k = reinterpret_cast<const char*>(a.k + (size_t)it.row0 * a.ld_k + (size_t)kvh * D);
    stage.v = reinterpret_cast<const char*>(a.v + (size_t)it.row0 * a.ld_v + (size_t)kvh * D);
    stage.ld_k = a.ld_k;
    stage.ld_v = a.ld_v;
  } else {
    stage.k = reinterpret_cast<const char*>(a.k);
    stage.v = reinterpret_cast<const char*>(a.v);
    stage.table = a.page_table + (size_t)it.seq * a.table_pages;
    stage.page_shift = a.page_shift;
    stage.n_pages = a.n_pages;
    stage.n_kv_heads = a.n_kv_heads;
  }
  TileRows<D> w;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const uint16_t* src = a.q + (size_t)(it.row0 + min(wave_row + 32 * b + col, it.rows - 1)) * a.ld_q + (size_t)head * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) w.q[b][ks] = *reinterpret_cast<const bf16x8*>(src + 16 * ks);
    w.m[b] = -INFINITY;
    w.l[b] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) w.acc[b][dt] = f32x16{};
  }
  const float scale = a.scale * kLog2e * (SRC == KV_PAGED_E4M3 ? a.k_scale[kvh] : 1.0f);
  if (threadIdx.x == 0) lds_again = 0;
  if (n_all > 0) {
    attend_tiles<D, SRC>(w, stage, 0, n, n_all, it.before + wave_row, last, scale);
    float test = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) test = fmaf(w.acc[b][dt][i], 0.0f, test);
    if (test != test) lds_again = 1;
    __syncthreads();
    if (uniform(lds_again)) attend_by_key<D, SRC>(w, stage, n_all, last, scale);
  }

#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int row = wave_row + 32 * b + col;
    const float l = w.l[b] + other_half(w.l[b]);
    if (row >= it.rows) continue;
    const float inv = l == 0.0f ? 0.0f : (SRC == KV_PAGED_E4M3 ? a.v_scale[kvh] : 1.0f) / l;
    uint16_t* dst = a.out + (size_t)(it.row0 + row) * a.ld_out + (size_t)head * D + 4 * half;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u32x2*>(dst + 32 * dt + 8 * i) =
            u32x2{pack2(w.acc[b][dt][4 * i] * inv, w.acc[b][dt][4 * i + 1] * inv), pack2(w.acc[b][dt][4 * i + 2] * inv, w.acc[b][dt][4 * i + 3] * inv)};
  }
}

template <int D>
hipError_t launch(const PromptArgs& a, int source, hipStream_t s) {
  const int group = a.n_heads / a.n_kv_heads, heads = group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1;
  // enough items for every way T rows can be shared out over the sequences
  const int64_t slots = (int64_t)a.T / (4 * kWaveRows / heads) + a.n_seqs, workgroups = slots * (a.n_heads / heads);
  if (workgroups > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 grid((unsigned)workgroups);
  if (source == KV_PACKED) k_attn_prompt<D, KV_PACKED><<<grid, kTileThreads, 0, s>>>(a, (int)slots, heads);
  else if (source == KV_PAGED) k_attn_prompt<D, KV_PAGED><<<grid, kTileThreads, 0, s>>>(a, (int)slots, heads);
  else k_attn_prompt<D, KV_PAGED_E4M3><<<grid, kTileThreads, 0, s>>>(a, (int)slots, heads);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attn_prompt(const PromptArgs& a, int source, hipStream_t s) {
  return a.head_dim == 128 ? launch<128>(a, source, s) : launch<64>(a, source, s);
}

}  // namespace mes
