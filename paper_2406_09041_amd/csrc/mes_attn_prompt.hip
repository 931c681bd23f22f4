// Causal attention over packed prompts, and over new tokens behind a paged cache.  Bound by the matrix cores (and the
// exponentials between their products); the mathematics, per query row with scores s_j = scale * <q, k_j>:
//   p_j = 2^(s_j log2e - m) with a bound m of the exponents, at most kSlack above the largest, l = sum p_j, o = sum p_j v_j / l
// in one pass over the keys, 64 at a time, nothing of the scores in memory (mes_attn_tiles.h).
//
// A workgroup is 4 wavefronts of 32 query rows: of up to 4 heads that share keys and values (all of them then see as many keys,
// and no wavefront waits for another), else of consecutive rows of one head.  Where some of these items see so many keys that they
// would work long after the others, the call is cut: the keys of every sequence in blocks, an item's part of a block is a workgroup's.
// The parts of a block run at about the same time, so that its keys and values come from HBM once and then from L2 (parts cut
// wherever an equal share ended asked for 4.2 TB/s of different tiles).  The parts of an item leave their sums in the workspace and
// k_join_prompt adds them up.  The lengths are on the device, so every workgroup finds its part by itself.
//
// Measured (head_dim 128, 32 heads over 8 key / value heads unless stated): one prompt of 77 rows 8.8 us, of which 7 is the time of a launch
// that does next to nothing; four of 1024 rows 53 us; 1 to 6001 rows of 40 heads with keys of their own 411 us, 961 TFLOP/s; 8
// prompts of 1 to 700 rows behind 0 to 4096 cached tokens 105 us, at e4m3 or over blocks 118 (widening the codes and writing them to LDS).
#include "mes_attn_cut.h"
#include "mes_attn_tiles.h"

namespace mes {
namespace {

static_assert(kTile == kCutTile, "tiles of keys");

// The part of the call a workgroup works on
struct Item {
  int seq, row0, rows, tile, before;   // sequence; its first row in the call; its rows; tile of R of them; tokens before row 0
};

template <int SRC>
__device__ __forceinline__ int rows_of(const PromptArgs& a, int s, int& lo) {
  lo = min(max(a.q_offsets[s], 0), a.T);
  return max(min(a.q_offsets[s + 1], a.T) - lo, 0);
}

// Tokens before the sequence's row `lo`, its first: all that the offsets name count, also those that the call does not have.  More than the table has room for makes no
// difference to any row.
__device__ __forceinline__ int tokens_before(const PromptArgs& a, int s, int lo) { return min(max(a.kv_len[s], 0) - max(a.q_offsets[s + 1] - lo, 0), a.capacity); }

// Up to 64 sequences: lane s looks after sequence s.  Keys are counted in units of R: item t of a sequence sees about base + t + 1.
struct Lanes {
  int lo, n, before, tiles, base;      // first row, rows, tokens before them; items; keys before the rows
  int all_items, longest;
  int block, parts, ahead, all_parts;  // units of a block (0: the call is not cut); parts of the sequence, and before it
};

// cut_slots: what the workspace has room for, 0: the call is not cut
template <int SRC>
__device__ Lanes look(const PromptArgs& a, int R, int columns, int cut_slots) {
  const int lane = threadIdx.x & 63;
  Lanes y = {};
  if (lane < a.n_seqs) {
    y.n = rows_of<SRC>(a, lane, y.lo);
    if (SRC != KV_PACKED) y.before = tokens_before(a, lane, y.lo);
  }
  y.tiles = (y.n + R - 1) / R;
  y.base = (max(y.before, 0) + R - 1) / R;
  y.all_items = wave_sum(y.tiles);
  y.longest = wave_max(y.tiles ? y.base + y.tiles : 0);
  if (cut_slots == 0 || y.all_items * columns > kMostCut) return y;
  const int block = cut_block(SRC == KV_PACKED, R, columns, y.all_items, y.longest, wave_sum(y.tiles * y.base + y.tiles * (y.tiles + 1) / 2));
  if (!block) return y;
  y.parts = y.tiles ? parts_below((y.base + y.tiles + block - 1) / block, block, y.base, y.tiles) : 0;
  // sequences in order of their longest rows
  for (int k = 0; k < a.n_seqs; ++k) {
    const int reach = __builtin_amdgcn_readlane(y.base + y.tiles, k), count = __builtin_amdgcn_readlane(y.parts, k);
    if (reach > y.base + y.tiles || (reach == y.base + y.tiles && k < lane)) y.ahead += count;
    y.all_parts += count;
  }
  y.block = y.all_parts * columns <= cut_slots ? block : 0;   // (offsets out of order can name more rows than the call has)
  return y;
}

__device__ __forceinline__ void pick(const Lanes& y, int s, int tile, Item& it) {
  it.seq = s;
  it.tile = tile;
  it.row0 = __builtin_amdgcn_readlane(y.lo, s);
  it.rows = __builtin_amdgcn_readlane(y.n, s);
  it.before = __builtin_amdgcn_readlane(y.before, s);
}

// Part j of a call that is cut; block: which block of keys.  The blocks of a sequence one after the other, so that its short parts
// (the last block of every item) come late.
__device__ bool part_number(const Lanes& y, int j, Item& it, int& block) {
  if (j >= y.all_parts) return false;
  const int s = __builtin_ctzll(__ballot(y.ahead <= j && j < y.ahead + y.parts));
  const int base = __builtin_amdgcn_readlane(y.base, s), tiles = __builtin_amdgcn_readlane(y.tiles, s), at = j - __builtin_amdgcn_readlane(y.ahead, s);
  int low = 0, high = (base + tiles - 1) / y.block;       // last block whose parts begin at or before this one
  while (low < high) {
    const int mid = (low + high + 1) >> 1;
    if (parts_below(mid, y.block, base, tiles) <= at) low = mid; else high = mid - 1;
  }
  block = low;
  pick(y, s, first_item(low, y.block, base) + at - parts_below(low, y.block, base, tiles), it);
  return true;
}

// Item j of a call that is not cut.  Up to 64 sequences: items in order of the keys they see, most first, so that no long one starts
// last.  More: tile t of sequence s has number floor(o[s] / R) + s + t, which leaves gaps (no item) but needs no sum over the
// sequences before it; the last first, as they see most of their sequence.
template <int SRC>
__device__ bool item_number(const PromptArgs& a, const Lanes& y, int R, int j, int slots, Item& it) {
  if (a.n_seqs <= 64) {
    const int lane = threadIdx.x & 63;
    if (j >= y.all_items) return false;
    // the level L with C(L + 1) <= j < C(L), C(L) = number of tiles with base + t >= L
    auto count = [&](int level) { return wave_sum(min(max(y.base + y.tiles - max(level, y.base), 0), y.tiles)); };
    int low = 0, high = y.longest;                        // C(low) > j >= C(high) = 0
    while (high - low > 1) {
      const int mid = low + (high - low) / 2;
      if (count(mid) > j) low = mid; else high = mid;
    }
    const int rank = j - count(low + 1);
    const bool mine = y.base <= low && low < y.base + y.tiles;
    const uint64_t who = __ballot(mine);
    const int s = __builtin_ctzll(__ballot(mine && __popcll(who & ((1ull << lane) - 1)) == rank));
    pick(y, s, low - __builtin_amdgcn_readlane(y.base, s), it);
    return true;
  }
  j = slots - 1 - j;
  if (j < 0) return false;
  int lo = 0, hi = a.n_seqs - 1;                           // last s with floor(o[s] / R) + s <= j
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (max(a.q_offsets[mid], 0) / R + mid <= j) lo = mid; else hi = mid - 1;
  }
  it.seq = lo;
  it.rows = rows_of<SRC>(a, lo, it.row0);
  it.tile = j - max(a.q_offsets[lo], 0) / R - lo;
  it.before = SRC != KV_PACKED ? tokens_before(a, lo, it.row0) : 0;
  return it.tile >= 0 && it.tile < (it.rows + R - 1) / R;
}

// The parts' results, per part and head group: (bound, sum) of the 128 rows of the wavefronts, and their weighted values in the order of the
// accumulators: [wavefront][4 dimensions: 8 (i / 4) + half][32 rows] x 4.
struct PieceLayout {
  size_t o, total;
};
__host__ __device__ inline PieceLayout piece_layout(int slots, int head_dim) {
  PieceLayout y;
  y.o = (size_t)slots * kTileWaves * kWaveRows * sizeof(float2);
  y.total = y.o + (size_t)slots * kTileWaves * kWaveRows * head_dim * sizeof(float);
  return y;
}

// Every row once more, key by key and with no key that it does not see: the way out where a value that some rows do not see is infinite
// or NaN (a weight of 0 times it is NaN, also in the rows that must not notice).
template <int D, int SRC>
__device__ __forceinline__ void attend_by_key(TileRows<D>& w, Stage<D, SRC>& stage, int first, int n_all, const int (&last)[NB], float scale) {
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
  for (int t = first; t < first + n_all; ++t) {
    barrier();                                                      // nobody reads the tiles of LDS any more
    stage.look_up(t);
    stage.request(t, 0);
    stage.deposit(t, 0);
    stage.request(t, 1);
    stage.deposit(t, 1);
    stage.template arrive<0>();
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
        const float raised = seen && dot > w.m[b] ? dot + kSlack : w.m[b];
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

// heads: heads of one workgroup (1, 2 or 4, a divisor of the heads per key / value head); slots: see item_number; cut_slots: what the
// workspace has room for (0: the call is not cut)
template <int D, int SRC>
__global__ __launch_bounds__(kTileThreads, 2) void k_attn_prompt(PromptArgs a, int slots, int heads, int cut_slots) {
  constexpr int KS = D / 16, DT = D / 32;
  __shared__ __align__(16) TileLds<D> lds;
  __shared__ int lds_again;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int R = kTileWaves * kWaveRows / heads, columns = a.n_heads / heads;  // rows of an item, workgroups of one item
  // consecutive workgroups go to the XCDs in turn: those that share keys and values come n_kv_heads apart, which puts them on
  // one XCD (8, 16, 40 ... key / value heads), whose L2 then fetches them once
  const int hx = blockIdx.x % columns, kvh = hx % a.n_kv_heads;
  const int head = kvh * (a.n_heads / a.n_kv_heads) + hx / a.n_kv_heads * heads + wave % heads;

  Item it;
  int block = 0, blocks = 1, block_keys = 0;                         // of the item's keys
  bool found;
  {
    Lanes y = {};
    if (a.n_seqs <= 64) y = look<SRC>(a, R, columns, cut_slots);
    if (uniform(y.block)) {
      found = part_number(y, blockIdx.x / columns, it, block);
      block = uniform(block);
      block_keys = uniform(y.block) * R;
      blocks = uniform(found ? ((max(it.before, 0) + R - 1) / R + it.tile) / y.block + 1 : 1);
    } else {
      found = item_number<SRC>(a, y, R, blockIdx.x / columns, slots, it);
    }
  }
  if (!uniform(found)) return;
  it.seq = uniform(it.seq); it.row0 = uniform(it.row0); it.rows = uniform(it.rows); it.tile = uniform(it.tile); it.before = uniform(it.before);
  const int row_first = it.tile * R;

  // keys [kTile first, kv_end) are seen by some row of the workgroup
  const int capacity = SRC == KV_PACKED ? 0x7fffffff : a.capacity;
  const int first = block * (block_keys / kTile), block_end = block + 1 < blocks ? (block + 1) * block_keys : 0x7fffffff;
  const int kv_end = uniform(min(min(it.before + min(row_first + R, it.rows), capacity), block_end));
  const int n_all = kv_end > first * kTile ? (kv_end + kTile - 1) / kTile - first : 0;
  const int wave_row = row_first + wave / heads * kWaveRows;         // the wavefront's first row
  const int high = min(it.before + min(wave_row + kWaveRows, it.rows), kv_end);     // keys seen by its last row
  const int n = wave_row < it.rows && high > first * kTile ? (high + kTile - 1) / kTile - first : 0;
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
    stage.exponents[0] = a.k_exponent;
    stage.exponents[1] = a.v_exponent;
    stage.n_pages = a.n_pages;
    stage.n_kv_heads = a.n_kv_heads;
  }
  const float factor = a.scale * kLog2e * (SRC == KV_PAGED_E4M3 ? a.k_scale[kvh] : 1.0f), scale = SRC == KV_PAGED_E4M3 ? factor_of_scores(factor) : factor;
  TileRows<D> w;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const uint16_t* src = a.q + (size_t)(it.row0 + min(wave_row + 32 * b + col, it.rows - 1)) * a.ld_q + (size_t)head * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) w.q[b][ks] = *reinterpret_cast<const bf16x8*>(src + 16 * ks);
    if constexpr (SRC == KV_PAGED_E4M3) factor_to_query(w.q[b], factor);
    w.m[b] = -INFINITY;
    w.l[b] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) w.acc[b][dt] = f32x16{};
  }
  if (threadIdx.x == 0) lds_again = 0;
  if (n_all > 0) {
    attend_tiles<D, SRC>(w, stage, first, n, n_all, it.before + wave_row, last, scale);
    float test = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) test = fmaf(w.acc[b][dt][i], 0.0f, test);
    if (test != test) lds_again = 1;
    __syncthreads();
    if (uniform(lds_again)) attend_by_key<D, SRC>(w, stage, first, n_all, last, scale);
  }

  if (blocks > 1) {
    const PieceLayout y = piece_layout(cut_slots, D);
    const int slot = blockIdx.x;
    char* ws = static_cast<char*>(a.ws);
    float2* ml = reinterpret_cast<float2*>(ws) + ((size_t)slot * kTileWaves + wave) * kWaveRows;
    f32x4* o = reinterpret_cast<f32x4*>(ws + y.o) + ((size_t)slot * kTileWaves + wave) * kWaveRows * (D / 4);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const float l = w.l[b] + other_half(w.l[b]);
      if (half == 0) ml[32 * b + col] = make_float2(w.m[b], l);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          o[((dt * 4 + i) * 2 + half) * kWaveRows + 32 * b + col] = f32x4{w.acc[b][dt][4 * i], w.acc[b][dt][4 * i + 1], w.acc[b][dt][4 * i + 2], w.acc[b][dt][4 * i + 3]};
    }
    return;
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

// Adds up the parts of the items that were cut.  A workgroup's job is 32 rows and 32 dimensions of an item, its wavefronts share out the
// blocks; blockIdx.x is (item, heads), blockIdx.y takes every gridDim.y-th job of it.
constexpr int kJoinThreads = 256;
template <int D, int SRC>
__global__ __launch_bounds__(kJoinThreads) void k_join_prompt(PromptArgs a, int heads, int cut_slots) {
  constexpr int kQuads = 4;                                          // groups of 4 dimensions x 2 halves per job
  __shared__ f32x4 part[4][kQuads][64];
  __shared__ float2 part_ml[4][64];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  const int R = kTileWaves * kWaveRows / heads, columns = a.n_heads / heads, hx = blockIdx.x % columns, kvh = hx % a.n_kv_heads;
  const int item = blockIdx.x / columns;
  const Lanes y = look<SRC>(a, R, columns, cut_slots);
  const int block = uniform(y.block);
  if (!block || item >= y.all_items) return;
  const int upto = wave_scan(y.tiles);                               // items up to and with the lane's
  const int s = __builtin_ctzll(__ballot(upto > item));
  const int tiles = __builtin_amdgcn_readlane(y.tiles, s), base = __builtin_amdgcn_readlane(y.base, s), tile = uniform(item - __builtin_amdgcn_readlane(upto, s) + tiles);
  const int blocks = (base + tile) / block + 1;
  if (blocks == 1) return;
  const int ahead = __builtin_amdgcn_readlane(y.ahead, s), row0 = __builtin_amdgcn_readlane(y.lo, s) + tile * R, rows = min(R, __builtin_amdgcn_readlane(y.n, s) - tile * R);
  const char* ws = static_cast<const char*>(a.ws);
  for (int job = blockIdx.y; job < kTileWaves * (D / 32); job += gridDim.y) {
    const int part_wave = job % kTileWaves, q0 = job / kTileWaves * kQuads, row = part_wave / heads * kWaveRows + col;
    if (part_wave / heads * kWaveRows >= rows) continue;
    const float2* ml = reinterpret_cast<const float2*>(ws) + part_wave * kWaveRows + col;
    const f32x4* o = reinterpret_cast<const f32x4*>(ws + piece_layout(cut_slots, D).o) + (part_wave * (D / 4) + 2 * q0 + half) * kWaveRows + col;
    float m = -INFINITY, l = 0.0f;
    f32x4 x[kQuads] = {};
    for (int p = wave; p < blocks; p += 4) {
      const int number = ahead + parts_below(p, block, base, tiles) + tile - first_item(p, block, base);
      const size_t slot = (size_t)number * columns + hx, step_ml = slot * kTileWaves * kWaveRows, step_o = step_ml * (D / 4);
      const float2 v = ml[step_ml];
      f32x4 r[kQuads];
#pragma unroll
      for (int q = 0; q < kQuads; ++q) r[q] = o[step_o + q * 2 * kWaveRows];
      const float raised = fmaxf(m, v.x), to = raised == -INFINITY ? 0.0f : raised;
      const float old = exp2_fast(m - to), f = exp2_fast(v.x - to);
      m = raised;
      l = l * old + v.y * f;
#pragma unroll
      for (int q = 0; q < kQuads; ++q) x[q] = x[q] * old + r[q] * f;
    }
    __syncthreads();
    part_ml[wave][lane] = make_float2(m, l);
#pragma unroll
    for (int q = 0; q < kQuads; ++q) part[wave][q][lane] = x[q];
    __syncthreads();
    // wavefront w finishes group w
    float top = -INFINITY, sum = 0.0f;
    f32x4 all = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, part_ml[w][lane].x);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = exp2_fast(part_ml[w][lane].x - (top == -INFINITY ? 0.0f : top));
      sum += part_ml[w][lane].y * f;
      all += part[w][wave][lane] * f;
    }
    if (row < rows) {
      const int head = kvh * (a.n_heads / a.n_kv_heads) + hx / a.n_kv_heads * heads + part_wave % heads;
      const float inv = sum == 0.0f ? 0.0f : (SRC == KV_PAGED_E4M3 ? a.v_scale[kvh] : 1.0f) / sum;
      uint16_t* dst = a.out + (size_t)(row0 + row) * a.ld_out + (size_t)head * D + 8 * (q0 + wave) + 4 * half;
      *reinterpret_cast<u32x2*>(dst) = u32x2{pack2(all[0] * inv, all[1] * inv), pack2(all[2] * inv, all[3] * inv)};
    }
  }
}

inline int heads_of(int group) { return group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1; }
// enough items for every way T rows can be shared out over the sequences
inline int64_t slots_of(int T, int n_seqs, int heads) { return (int64_t)T / (kTileWaves * kWaveRows / heads) + n_seqs; }
// Whether look() could cut a call of packed prompts whose sequences take up all T rows: for some length of the longest, the others
// sharing the rest evenly, which is the least work there can be beside it.  (Where it could not, there is no launch that finds nothing to join.)
bool packed_may_cut(int T, int n_seqs, int R, int columns) {
  const int rows = (T + R - 1) / R;
  for (int longest = (rows + n_seqs - 1) / n_seqs;; longest += longest / 10 + 1) {
    longest = std::min(longest, rows);
    const int others = n_seqs - 1, rest = rows - longest, each = others ? (rest + others - 1) / others : 0;
    const int64_t units = ((int64_t)longest * (longest + 1) + (others ? (int64_t)rest * rest / others + rest : 0)) / 2;
    if (cut_block(true, R, columns, std::max(longest, rows), std::max(longest, each), (int)std::min<int64_t>(units, 1 << 28))) return true;
    if (longest == rows) return false;
  }
}

template <int D>
hipError_t launch(const PromptArgs& a, int source, hipStream_t s) {
  const int heads = heads_of(a.n_heads / a.n_kv_heads), columns = a.n_heads / heads;
  const int64_t slots = slots_of(a.T, a.n_seqs, heads), workgroups = slots * columns;
  if (workgroups > 0xffffff) return hipErrorInvalidValue;
  // not cut: where no item can be much longer than the shortest part; with capacities at which the line would pass 31 bits
  const int longest = source == KV_PACKED ? a.T : a.capacity;
  const bool cut = a.ws && a.n_seqs <= 64 && columns <= kHeld && longest > 11 * kTile && longest <= 1 << 24 &&
                   (source != KV_PACKED || packed_may_cut(a.T, a.n_seqs, kTileWaves * kWaveRows / heads, columns));
  const int cut_slots = cut ? cut_slots_of(workgroups) : 0;
  const dim3 grid((unsigned)std::max<int64_t>(workgroups, cut_slots / columns * columns));
  // joining workgroups: enough to fill the chip where there are few items
  const int64_t items = std::min<int64_t>(workgroups, kMostCut);
  const dim3 join((unsigned)items, (unsigned)std::max<int64_t>(1, std::min<int64_t>(kTileWaves * (D / 32), 2048 / items)));
  auto go = [&](auto src) {
    constexpr int SRC = decltype(src)::value;
    k_attn_prompt<D, SRC><<<grid, kTileThreads, 0, s>>>(a, (int)slots, heads, cut_slots);
    if (cut) k_join_prompt<D, SRC><<<join, kJoinThreads, 0, s>>>(a, heads, cut_slots);
  };
  if (source == KV_PACKED) go(std::integral_constant<int, KV_PACKED>{});
  else if (source == KV_PAGED) go(std::integral_constant<int, KV_PAGED>{});
  else if (source == KV_PAGED_E4M3) go(std::integral_constant<int, KV_PAGED_E4M3>{});
  else go(std::integral_constant<int, KV_PAGED_BLOCKS>{});
  return hipGetLastError();
}

}  // namespace

size_t attn_prompt_workspace_bytes(int T, int n_seqs, int n_heads, int n_kv_heads, int head_dim) {
  const int heads = heads_of(n_heads / n_kv_heads);
  return piece_layout(cut_slots_of(slots_of(T, n_seqs, heads) * (n_heads / heads)), head_dim).total;
}

hipError_t launch_attn_prompt(const PromptArgs& a, int source, hipStream_t s) {
  return a.head_dim == 128 ? launch<128>(a, source, s) : launch<64>(a, source, s);
}

}  // namespace mes
