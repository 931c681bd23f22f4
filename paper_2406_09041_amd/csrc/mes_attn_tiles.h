// Many query rows against keys and values that a workgroup shares in LDS: the loop of the prompt kernel, and of the decode
// kernel where many rows read the same tokens.
//
// A workgroup is 4 wavefronts of 32 query rows; keys come 64 at a time.  Scores are formed transposed, S^T = K Q^T: in the
// result of v_mfma_f32_32x32x16_bf16 a lane holds ONE query row (lane & 31) and 16 of 32 keys, so that maxima, sums and rescaling
// need no exchange but one with lane ^ 32, and its registers, rounded to bf16, ARE the operand P^T of the second product
// O^T = V^T P^T: keys 4 h + (0..3) and 8 + 4 h + (0..3) of every 16 for half h of the wavefront.  V's operand for these keys is read
// from LDS with the transposing read (ds_read_b64_tr_b16), in P's order of keys.
//
// Matrix cores and vector units are kept busy together: while the scores of tile t + 1 are multiplied, the exponentials of tile t are
// formed between the products, and while tile t is multiplied with V, the maxima of tile t + 1.  The groups of an operand read, a
// product and the vector work that goes with them are kept in this order by scheduling barriers; operands are read three groups ahead.
//
// Why 32 rows and two wavefronts per SIMD: with 64 rows an operand read from LDS serves two products, but one wavefront per
// SIMD with all 512 registers stood still at every barrier and every rescaling; two of 32 rows fill each other's gaps.  Measured at head_dim
// 128: 40 heads of prompts of 1 to 6001 rows 411 us, 961 TFLOP/s of the 1268 that a bf16 library product of 8192^3 reaches on the same
// card; one prompt of 8192 rows of 32 heads 1083.  What bounds it: the exponentials and sums take about as many issue slots as the
// products take matrix cycles, and what the scheduler cannot lay beside each other is lost.
//
// LDS: rows of head_dim, two tiles of keys and two of values in turn.  A copy of a wavefront writes 1 KiB in the order of its lanes: a
// block of 4 (8) rows, whose 16-byte pieces are XORed with turn(row) by fetching them in that order, and blocks are 16 bytes further
// apart than they are long.  Together this spreads both the 16 rows that a K operand reads at one piece and the 4 rows x 64 bytes
// of a transposing read over all banks; the rows of a block decide the XOR, so that an operand's address is one of 4 per lane plus
// a constant.
#pragma once

#include "mes_attn_common.h"

namespace mes {

constexpr int kTile = 64, kRing = 2, kTileWaves = 4, kTileThreads = 64 * kTileWaves, NB = 1, kWaveRows = 32 * NB;
constexpr int kPart = kTile / kTileWaves;                             // keys of a tile that a wavefront brings

constexpr int kBlock = 1024 + 16;                                     // bytes between blocks of rows

template <int D>
struct Row {
  static constexpr int kBytes = D * 2, kPieces = D / 8, kPerBlock = 64 / kPieces;
  // what the pieces of row r are XORed with
  static __device__ __forceinline__ int turn(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2 | ((r >> 2) & 1) << 1; }
  static constexpr __host__ __device__ int at(int r) { return r / kPerBlock * kBlock + r % kPerBlock * kBytes; }
};

template <int D>
struct TileLds {
  static constexpr int kTileBytes = kTile / Row<D>::kPerBlock * kBlock;
  char kv[2][kRing][kTileBytes];      // keys, values
};

// What an absent token (behind the sequence's end, before the first that is seen, or on a page that does not exist) is read from: its value
// row must not be able to turn a weight of 0 into NaN.
static __device__ const u32x4 g_zeros[16] = {};

// 16 bytes per lane, lane l's to LDS address `to` + 16 l.  Written as instructions: for its builtin the compiler would make every
// later LDS access of the wavefront wait for the copy, as it cannot tell that nobody reads that tile yet.
__device__ __forceinline__ void copy_to_lds(const void* from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(to) : "memory", "m0");
}
// base: the same in all lanes.  A vector instruction may have written its registers just before (a value that was kept in a lane), and a
// vector memory instruction must not read such a register for 5 wait states, which the compiler does not look after in here: a scalar
// copy of it may be read at once, and takes the place of the wait that M0 needs.
__device__ __forceinline__ void copy_to_lds(const void* base, uint32_t offset, uint32_t to) {
  const void* at;
  asm volatile("s_mov_b32 m0, %3\n\ts_mov_b64 %0, %2\n\tglobal_load_lds_dwordx4 %1, %0" : "=&s"(at) : "v"(offset), "s"(base), "s"(to) : "memory", "m0");
}

// LDS accesses of the wavefront are done, then everybody's; copies into LDS are waited for apart.
__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Brings tiles of keys and values to LDS.  Wavefront w brings keys 16 w .. 16 w + 15 of every tile; the copies write 16 bytes per
// lane in order, so the turn is applied to the address that a lane fetches.  Key j of the tiles is token j of the sequence.
template <int D, int SRC>
struct Stage {
  static constexpr int kPieces = Row<D>::kPieces, kRowsCopy = Row<D>::kPerBlock, kCopies = kPart / kRowsCopy;
  const char *k, *v;              // packed: the sequence's row 0 of this head; paged: the cache's layer
  int ld_k, ld_v;                 // packed: elements between rows
  const int32_t* table;           // paged: the sequence's page table
  int page_shift, n_pages, n_kv_heads, kvh;
  int first, from, to;            // the first tile; tokens [from, to) are seen
  TileLds<D>& lds;
  int lane, wave;
  uint32_t offset[2];             // of a lane's 16 bytes from the first row of its copy
  static constexpr bool kCodes = SRC == KV_PAGED_E4M3 || SRC == KV_PAGED_BLOCKS;
  int pages[4], batch;            // pages of the 16-token parts of tiles batch .. batch + 63, one tile per lane
  const uint8_t* exponents[2];    // blocks: of the cache's layer, keys and values
  int exponent[2];                // of the wavefront's part, one tile per lane
  static constexpr int kLanes = 64 / kPart, kWords = D / kLanes / 4;   // codes: lanes per key, words of codes of a lane
  u32x4 raw[kWords / 4];          // codes on their way

  __device__ Stage(TileLds<D>& l) : ld_k(D), ld_v(D), from(0), lds(l), lane(threadIdx.x & 63), wave(uniform(threadIdx.x >> 6)), batch(-64) {}
  __device__ __forceinline__ void begin(int tile) {
    first = tile;
    const int r = lane / kPieces;
    const uint32_t piece = ((lane % kPieces) ^ Row<D>::turn(r)) * 16;
    offset[0] = (uint32_t)r * ld_k * 2 + piece;
    offset[1] = (uint32_t)r * ld_v * 2 + piece;
  }
  __device__ __forceinline__ char* slot(int tile, int kv) { return lds.kv[kv][(tile - first) % kRing]; }

  __device__ __forceinline__ void look_up(int tile) {
    if constexpr (SRC != KV_PACKED) {
      if (tile >= batch && tile < batch + 64) return;
      batch = max(tile - 3, 0);                                      // the tiles before it are still asked about
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t token = (int64_t)(batch + lane) * kTile + 16 * i;
        pages[i] = token < to ? table[token >> page_shift] : -1;
      }
      if constexpr (SRC == KV_PAGED_BLOCKS) {
        static_assert(kPart == MES_KV_BLOCK && kTileWaves == 4, "a wavefront's part of a tile is a block");
        const int page = wave == 0 ? pages[0] : wave == 1 ? pages[1] : wave == 2 ? pages[2] : pages[3];
        const int slot = (int)((int64_t)(batch + lane) * kTile + kPart * wave) & ((1 << page_shift) - 1);
        const size_t at = block_at((unsigned)page < (unsigned)n_pages ? page : 0, kvh, n_kv_heads, page_shift, slot);
#pragma unroll
        for (int i = 0; i < 2; ++i) exponent[i] = exponent_of(exponents[i][at]);
      }
    }
  }
  __device__ __forceinline__ int page_of(int tile, int part) { return __builtin_amdgcn_readlane(pages[part], tile - batch); }
  // bit i: the 16 keys of part i have a page
  __device__ __forceinline__ int there(int tile) {
    if constexpr (SRC == KV_PACKED) return 15;
    int bits = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) bits |= ((unsigned)page_of(tile, i) < (unsigned)n_pages ? 1 : 0) << i;
    return bits;
  }
  // kv: 0 keys, 1 values
  __device__ __forceinline__ void request(int tile, int kv) {
    const int token0 = tile * kTile + kPart * wave;
    const char* base = kv ? v : k;
    const int step = (SRC == KV_PACKED ? (kv ? ld_v : ld_k) : D) * (kCodes ? 1 : 2);   // bytes between rows
    bool real = true;
    if constexpr (SRC == KV_PACKED) {
      base += (int64_t)token0 * step;
    } else {
      const int part = wave * kPart / 16;
      int page = part == 0 ? page_of(tile, 0) : part == 1 ? page_of(tile, 1) : part == 2 ? page_of(tile, 2) : page_of(tile, 3);
      real = (unsigned)page < (unsigned)n_pages;
      if (!real) page = 0;
      base += ((((int64_t)page * n_kv_heads + kvh) << page_shift) + (token0 & ((1 << page_shift) - 1))) * step;
    }
    const bool lead = from > 0 && token0 < from;                      // never in the prompt kernel, where `from` is 0
    if constexpr (!kCodes) {
      const uint32_t at = (uint32_t)(uintptr_t)slot(tile, kv) + Row<D>::at(kPart * wave);
      if (real && !lead && token0 + kPart <= to) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) copy_to_lds(base + (int64_t)i * kRowsCopy * step, offset[kv], at + i * kBlock);
      } else {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const int token = token0 + i * kRowsCopy + lane / kPieces;
          const bool there = real && token < to && !(lead && token < from);
          copy_to_lds(there ? (const void*)(base + (int64_t)i * kRowsCopy * step + offset[kv]) : (const void*)&g_zeros[lane % kPieces], at + i * kBlock);
        }
      }
    } else {
      const int r = lane / kLanes;
      const char* codes = base + (uint32_t)(r * D + lane % kLanes * (D / kLanes));
      const bool there = real && token0 + r < to && !(lead && token0 + r < from);
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) raw[i] = there ? *reinterpret_cast<const u32x4*>(codes + 16 * i) : u32x4{0, 0, 0, 0};
    }
  }
  // all of this wavefront's copies but the last `younger`
  template <int younger>
  __device__ __forceinline__ void arrive() {
    if constexpr (!kCodes) asm volatile("s_waitcnt vmcnt(%0)" : : "n"(younger) : "memory");
  }
  __device__ __forceinline__ void deposit(int tile, int kv) {        // codes -> bf16 rows in LDS
    if constexpr (kCodes) {
      const float power = SRC == KV_PAGED_BLOCKS ? power_of(__builtin_amdgcn_readlane(exponent[kv], tile - batch)) : 1.0f;
      const int r = kPart * wave + lane / kLanes, piece = lane % kLanes * (kWords / 2);
#pragma unroll
      for (int i = 0; i < kWords / 2; ++i) {
        const u32x2 x = widen4(raw[i / 2][2 * (i % 2)], power), y = widen4(raw[i / 2][2 * (i % 2) + 1], power);
        *reinterpret_cast<u32x4*>(slot(tile, kv) + Row<D>::at(r) + (((piece + i) ^ Row<D>::turn(r)) * 16)) = u32x4{x[0], x[1], y[0], y[1]};
      }
    }
  }
};

template <int D>
struct TileRows {
  static constexpr int KS = D / 16, DT = D / 32;
  bf16x8 q[NB][KS];               // NB = 1 block of 32 rows; Q^T operands: lane (col, half) holds dimensions 16 ks + 8 half + (0..7) of row col of the block
  f32x16 acc[NB][DT];             // O^T: lane holds its row, dimensions 32 dt + 8 (i / 4) + 4 half + i % 4
  float m[NB], l[NB];              // running bound of the scores (in powers of two); sum over this half's keys
};

// One tile's scores -> -inf where the row does not see the key.  `last[b]`: the last key that the lane's row of block b sees.
__device__ __forceinline__ void mask_scores(f32x16 (&s)[NB][2], int key0, const int (&last)[NB], int from, int to, int there) {
  const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int limit = min(last[b], to - 1) - key0 - 4 * half;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (32 * tt + 8 * (i / 4) + i % 4 > limit) s[b][tt][i] = -INFINITY;
  }
  if (key0 < from) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * tt + 8 * (i / 4) + i % 4 < from - key0 - 4 * half) s[b][tt][i] = -INFINITY;
  }
  if (there == 15) return;
#pragma unroll
  for (int part = 0; part < 4; ++part)
    if (!((there >> part) & 1)) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 8; ++i) s[b][part / 2][8 * (part % 2) + i] = -INFINITY;
    }
}

// Tiles [first, first + n) of this wavefront's rows, of the workgroup's [first, first + n_all) (n <= n_all), keys up to stage.to; no row sees a key
// behind the last tile.  low: the last key that the row
// seeing least sees; last: see mask_scores.  Every wavefront of the workgroup makes the call; LDS is free before it.
template <int D, int SRC>
__device__ __forceinline__ void attend_tiles(TileRows<D>& w, Stage<D, SRC>& stage, int first, int n, int n_all, int low, const int (&last)[NB], float scale) {
  constexpr int KS = D / 16, DT = D / 32;
  constexpr int kGroups1 = 2 * KS, kGroups2 = 4 * DT;               // groups of two products: scores, values
  constexpr int kPairs = 16 * NB / kGroups1;                             // pairs of weights formed per group of scores
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  TileLds<D>& lds = stage.lds;

  // operands from LDS
  typedef __attribute__((address_space(3))) char* lds_char;
  typedef __attribute__((address_space(3))) bf16x8* lds_b128;
  typedef __attribute__((address_space(3))) i16x4* lds_tr;
  typedef Row<D> R;
  const lds_char base = (lds_char)&lds.kv[0][0][0];
  constexpr int kTileBytes = TileLds<D>::kTileBytes, kTogether = D / 64;   // kTogether: neighbouring pieces that a turn leaves neighbours, / 2
  const int v_r = 4 * half + ((lane & 15) >> 2);
  uint32_t k_at[4], v_at[DT];
#pragma unroll
  for (int i = 0; i < 4; ++i) k_at[i] = R::at(col) + (((2 * kTogether * i + half) ^ R::turn(col)) * 16);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) v_at[dt] = R::at(v_r) + (((4 * dt + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ R::turn(v_r)) * 16) + 8 * (lane & 1);
  auto k_operand = [&](int g) {                                     // group g: dimensions 16 (g / 2) .., keys 32 (g % 2) ..
    const int ks = g / 2;
    return *(lds_b128)(base + k_at[ks / kTogether] + (R::at(32 * (g % 2)) + ks % kTogether * 32));
  };
  auto v_operand = [&](int g) {                                     // group g: keys 16 (g / DT) .., dimensions 32 (g % DT) ..
    // lanes of 16 read 4 keys x 16 dimensions, 8 bytes each, and get a dimension's 4 keys
    const int at = kRing * kTileBytes + R::at(16 * (g / DT));
    struct { i16x4 lo, hi; } v;
    v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)(base + v_at[g % DT] + at));
    v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_tr)(base + v_at[g % DT] + at + R::at(8)));
    return __builtin_bit_cast(bf16x8, v);
  };
  // the addresses move on to the next tile of the ring
  auto next_k = [&](int tile) {
    const uint32_t by = (tile - first) % kRing == 0 ? (uint32_t)(-(kRing - 1) * kTileBytes) : (uint32_t)kTileBytes;
#pragma unroll
    for (int i = 0; i < 4; ++i) k_at[i] += by;
  };
  auto next_v = [&](int tile) {
    const uint32_t by = (tile - first) % kRing == 0 ? (uint32_t)(-(kRing - 1) * kTileBytes) : (uint32_t)kTileBytes;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) v_at[dt] += by;
  };

  f32x16 s0[NB][2], s1[NB][2];                                        // scores [block][32 keys] of two tiles in turn
  float from[NB];

  auto raise = [&](const float (&top)[NB]) {                          // the bounds, seldom
    bool above = false;
#pragma unroll
    for (int b = 0; b < NB; ++b) above |= top[b] * scale > w.m[b];
    if (__any(above)) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const float t = fmaxf(top[b], other_half(top[b])) * scale;
        const float raised = fmaxf(w.m[b], t + kSlack);
        const float shrink = exp2_fast(w.m[b] - (raised == -INFINITY ? 0.0f : raised));
        w.l[b] *= shrink;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
          for (int i = 0; i < 16; ++i) w.acc[b][dt][i] *= shrink;
        w.m[b] = raised;
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) from[b] = w.m[b] == -INFINITY ? 0.0f : w.m[b];
  };
  auto partial = [&](int tile, int there) { return tile * kTile + kTile - 1 > low || tile * kTile + kTile > stage.to || tile * kTile < stage.from || there != 15; };

  // ---- keys run one tile ahead of the values: at tile t keys t + 1 and values t are needed, keys t + 2 and values t + 1 asked for (a ring of
  // three tiles and 8 wavefronts, which ask for them a tile earlier, measured the same).  Codes of an 8-bit cache pass through registers:
  // keys t + 2 during the first half of the work on tile t, values t + 1 during the second.
  const int end_all = first + n_all, end = first + n;
  constexpr bool kDirect = !Stage<D, SRC>::kCodes;
  auto before = [&](int t) {
    stage.template arrive<0>();
    barrier();                                                       // nobody reads keys t and values t - 1 any more
    if (t + 2 < end_all) {
      stage.look_up(t + 2);
      stage.request(t + 2, 0);
    }
    if (kDirect && t + 1 < end_all) stage.request(t + 1, 1);
  };
  auto between = [&](int t) {
    if (t + 2 < end_all) stage.deposit(t + 2, 0);
    if (!kDirect && t + 1 < end_all) stage.request(t + 1, 1);
  };
  auto after = [&](int t) {
    if (t + 1 < end_all) stage.deposit(t + 1, 1);
  };

  // Tile t, whose scores are in s; the scores of tile t + 1 go to sn.  Where there is none its scores are of what LDS holds, and all
  // masked: a step of its own for the last tile is more code, and code is fetched when it is first run.
  auto step = [&](f32x16 (&s)[NB][2], f32x16 (&sn)[NB][2], int t) {
    next_k(t + 1);
    if (t > first) next_v(t);
    u32x4 p[NB][4];
    constexpr int kAhead = kDirect ? 3 : 2;            // operands on their way; codes of the 8-bit cache need the registers
    bf16x8 ring[kAhead + 1];
#pragma unroll
    for (int g = 0; g < kAhead; ++g) ring[g] = k_operand(g);
#pragma unroll
    for (int g = 0; g < kGroups1; ++g) {
      ring[(g + kAhead) % (kAhead + 1)] = g + kAhead < kGroups1 ? k_operand(g + kAhead) : v_operand(g + kAhead - kGroups1);
      const f32x16 zero = {};
#pragma unroll
      for (int b = 0; b < NB; ++b)
        sn[b][g % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[g % (kAhead + 1)], w.q[b][g / 2], g < 2 ? zero : sn[b][g % 2], 0, 0, 0);
#pragma unroll
      for (int x = 0; x < kPairs; ++x) {
        const int i = (g * kPairs + x) % 4, b = (g * kPairs + x) / 4 % NB, st = (g * kPairs + x) / (4 * NB), e = 8 * (st % 2) + 2 * i;
        p[b][st][i] = pack2(exp2_fast(s[b][st / 2][e] * scale - from[b]), exp2_fast(s[b][st / 2][e + 1] * scale - from[b]));
        w.l[b] = add_pair(p[b][st][i], w.l[b]);                     // the sum of what is multiplied with V
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // the weights are needed behind the branches only, and would be formed there, with no products beside them
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int st = 0; st < 4; ++st) asm volatile("" : "+v"(p[b][st]));
    between(t);
    const int there = stage.there(t + 1);
    if (partial(t + 1, there)) mask_scores(sn, (t + 1) * kTile, last, stage.from, stage.to, there);
    float top[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) top[b] = -INFINITY;
#pragma unroll
    for (int g = 0; g < kGroups2; ++g) {
      if (g + kAhead < kGroups2) ring[(kGroups1 + g + kAhead) % (kAhead + 1)] = v_operand(g + kAhead);
#pragma unroll
      for (int b = 0; b < NB; ++b)
        w.acc[b][g % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[(kGroups1 + g) % (kAhead + 1)], __builtin_bit_cast(bf16x8, p[b][g / DT]), w.acc[b][g % DT], 0, 0, 0);
      constexpr int kEach = 32 * NB / kGroups2;                     // maxima per group
#pragma unroll
      for (int x = 0; x < kEach; ++x) {
        const int e = g * kEach + x;
        top[e / 32] = fmaxf(top[e / 32], sn[e / 32][e / 16 % 2][e % 16]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    raise(top);
  };

  stage.begin(first);
  stage.look_up(first);
  stage.request(first, 0);
  stage.deposit(first, 0);
  stage.request(first, 1);
  stage.deposit(first, 1);
  if (n_all > 1) {
    stage.request(first + 1, 0);
    stage.deposit(first + 1, 0);
  }
  // the first keys are there
  if (kDirect && n_all > 1) stage.template arrive<2 * Stage<D, SRC>::kCopies>(); else stage.template arrive<0>();
  barrier();
  if (n > 0) {
    const f32x16 zero = {};
#pragma unroll
    for (int g = 0; g < kGroups1; ++g) {
      const bf16x8 k = k_operand(g);
#pragma unroll
      for (int b = 0; b < NB; ++b) s0[b][g % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, w.q[b][g / 2], g < 2 ? zero : s0[b][g % 2], 0, 0, 0);
    }
    const int there = stage.there(first);
    if (partial(first, there)) mask_scores(s0, first * kTile, last, stage.from, stage.to, there);
    float top[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) top[b] = -INFINITY;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 16; ++i) top[b] = fmaxf(top[b], s0[b][tt][i]);
    raise(top);
  }
  int t = first;
  for (; t < end; t += 2) {                                          // one way out of the loop: with two, the compiler keeps two sets of accumulators
    before(t);
    step(s0, s1, t);
    after(t);
    if (t + 1 < end) {
      before(t + 1);
      step(s1, s0, t + 1);
      after(t + 1);
    }
  }
  t = end;
  for (; t < end_all; ++t) {                                         // other wavefronts' tiles
    before(t);
    between(t);
    after(t);
  }
}

}  // namespace mes
