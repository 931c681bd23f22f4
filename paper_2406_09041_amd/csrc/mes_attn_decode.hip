// One token of every sequence against the paged cache, prefixes that an expert's sequences share read once.  Bound by HBM:
// every distinct cached token is read once, 2 head_dim values per key / value head, for 4 head_dim n_heads operations.
//
// Work is a flat line of units (kUnit = 128 tokens of one key / value head): per key / value head first the shared
// prefixes (once per pass of up to 128 query rows), then what every sequence has of its own.  The line is cut into equal
// chunks, one per workgroup, wherever that falls: the workgroups are equally busy however the lengths are spread, also for one long
// sequence, and the launch does not depend on the lengths, which stay on the device (every workgroup adds them up for itself).  A
// piece of the line that does not cover a sequence alone leaves (bound, sum, weighted values) in the workspace, and k_join
// adds the pieces of a row in their order.
//
// Up to 16 query rows (one sequence of a group of up to 16 heads, or few sequences' shared prefix): a wavefront takes 32 tokens at a
// time.  Scores are formed transposed, S^T = K Q^T with v_mfma_f32_16x16x32_bf16: K's operand is 16 tokens x 8 dimensions per lane
// straight from memory, and the result holds one query row (lane & 15) and tokens 4 g + (0..3) per lane (g = lane / 16), which rounded
// to bf16 IS the operand P^T of O^T = V^T P^T over the 32 tokens in the order (4 g + i, 16 + 4 g + i).  V is read by rows, 16 lanes a
// row, lane r the dimensions VD r .. VD r + VD - 1 of its 8 tokens: product j of VD then yields the dimensions VD m + j, and its operand
// is pairs of 16-bit halves put together, one v_perm each.  So neither keys nor values pass through LDS.  Of the 16 columns of a
// tile 4 (n_heads / n_kv_heads) are used where nothing is shared: the matrix cores are idle most of the time anyway.
//
// More rows: up to 128 of them share keys and values in LDS (mes_attn_tiles.h), bound by the matrix cores from about 100 rows on.  The crossover
// at 16 rows is where the small body would read the tokens a second time: 64 sequences of 16 experts (1 to 25 each) took 62 us by passes of
// 16 rows and 47 through LDS, 96 behind one e4m3 prefix 94 and 60.
//
// Weights are rounded to bf16 for the product with V, as the matrix cores take both operands alike, and summed as rounded: they still add up
// to 1, and a row's error grows by at most 2^-8 of its weighted values' size (measured against 64 bits: 0.0020 of the rows' norm, 0.0017
// with weights in fp32).
//
// Measured (head_dim 128, 32 heads over 8 key / value heads): 256 sequences of 0 to 8192 tokens 160 us, 5.0 TB/s of the 5.96 that a
// pass that only reads reaches; the same at e4m3 99 us, 4.0 TB/s; 64 sequences of 512 tokens 26.5 us (5.1 TB/s); 64 of 16 experts with prompts of 512 to
// 1600 tokens 42 us, 106 MB; 96 behind 8200 shared tokens of an e4m3 cache 54 us, of which 10 us are products at the library's rate; one sequence of
// 200 tokens 8.3 us.  Own pieces cost 4 to 5 us each beside the larger body; in a launch of their own it was worse: 43 -> 51 us for the 64
// sequences, 59 -> 68 for the shared prefix.
#include "mes_attn_tiles.h"

namespace mes {
namespace {

constexpr int kThreads = 256, kUnit = 128, kRowsPass = 128, kFewRows = 16;
// Workgroups of a launch: what the chip holds.  Without shared prefixes and with up to 16 heads per key / value head only the small body is
// needed, which leaves room for three per compute unit (256 sequences of 0 to 8192 tokens, when it was made: 168 us, as a part
// of the larger kernel, two per compute unit, 186).
constexpr int kWorkgroups = 512, kWorkgroupsFew = 768;
// Up to this many tokens a sequence is one workgroup's, where nothing is shared: no second launch to add up pieces (one
// sequence of 200 tokens, when it was made: 9.2 us, 12.4 with it).
constexpr int kWholeTokens = 512;
static_assert(kThreads == kTileThreads && kRowsPass == kTileWaves * kWaveRows, "the workgroups of both bodies are the same");

struct Shape {                       // what host and device derive alike
  int group, per_pass, n_passes;     // query heads per key / value head, sequences per pass, passes of all groups
};

// partial results: [slot][rows][D] floats, then [slot][rows] (bound, sum)
struct Partials {
  float* o;
  float2* ml;
};

struct Layout {
  size_t prefix_o, prefix_ml, own_o, own_ml, meta, total;
};

__host__ __device__ inline Layout layout(int n_seqs, int n_kv_heads, int group, int n_passes, int head_dim) {
  const size_t pre = (size_t)(n_passes ? kWorkgroups + n_kv_heads * n_passes : 0) * kRowsPass;
  const size_t own = (size_t)(kWorkgroupsFew + n_kv_heads * n_seqs) * group;
  Layout y;
  y.prefix_o = 0;
  y.own_o = y.prefix_o + pre * head_dim * 4;
  y.prefix_ml = y.own_o + own * head_dim * 4;
  y.own_ml = y.prefix_ml + pre * 8;
  y.meta = (y.own_ml + own * 8 + 15) & ~(size_t)15;
  y.total = y.meta + (size_t)n_kv_heads * n_seqs * sizeof(int4);
  return y;
}

// where a (key / value head, sequence) finds its pieces: x first slot of its own part, y their number (-1: the row is
// written already), z first slot of the shared prefix, w number of those | row in the pass << 16
typedef int4 Meta;

struct DecodeCall {
  DecodeArgs a;
  Shape sh;
  int pass_base[MES_MAX_EXPERTS];
};

constexpr bool has_codes(int source) { return source != KV_PAGED; }

template <int D, int SRC>
struct Raw {                                        // 32 tokens of keys and values on their way
  static constexpr bool FP8 = has_codes(SRC);
  static constexpr int VD = D / 16, KC = FP8 ? D / 64 : D / 32, VW = VD * (FP8 ? 1 : 2) / 4;
  u32x4 k[2][KC];
  uint32_t v[8][VW];
};

// first dimension of the 8 that a lane holds in product c of K Q^T
template <int D, int SRC>
__device__ __forceinline__ int dim_of(int c, int g) {
  return has_codes(SRC) ? 64 * (c / 2) + 16 * g + 8 * (c % 2) : 32 * c + 8 * g;
}

struct Segment {                                    // a piece of the line
  int kvh, seq, seq0, rows;                         // key / value head; page table; sequence of row 0; query rows
  int from, to, t0, t1;                             // tokens of [from, to) in the units [t0, t1), t0 a multiple of 64
};

struct Nothing {};
template <int D, bool MANY>
struct Shared {
  union {
    std::conditional_t<MANY, TileLds<D>, Nothing> tiles;
    struct {
      float merge[4][kFewRows][D + 4];
      float2 ml[4][kFewRows];
    };
  };
  int cum[MES_MAX_SEQS + MES_MAX_EXPERTS + 1];
  int group_src[MES_MAX_EXPERTS];                   // first sequence as long as the prefix, -1: fewer than two are
  int part[4];
};

// The weighted sum over a piece with up to 16 query rows.  Pieces follow one another without a pause: a wavefront asks for the next piece's
// first tokens where it would ask for more of this one's, and knows their pages by then.
template <int D, int SRC>
struct Few {
  static constexpr bool FP8 = has_codes(SRC), SCALED = SRC == KV_PAGED_E4M3, BLOCKS = SRC == KV_PAGED_BLOCKS;
  static constexpr int VD = D / 16, KS = D / 32;
  typedef Raw<D, SRC> R;
  const DecodeArgs& a;
  int group, lane, wave, col, quad;
  u32x4 q[KS];                                      // Q^T operands
  R raw;                                            // the step that comes next
  int there[2];                                     // its pages
  int pages[2];                                     // of 64 steps of the piece, one step per lane
  int exponents[2][2];                              // blocks: of keys and values on these pages

  __device__ Few(const DecodeArgs& args, int g) : a(args), group(g), lane(threadIdx.x & 63), wave(uniform(threadIdx.x >> 6)), col(lane & 15), quad(lane >> 4) {}

  __device__ __forceinline__ int steps(const Segment& g) const { return ((g.t1 - g.t0 + 31) / 32 - wave + 3) / 4; }   // steps wave, wave + 4, ...
  __device__ __forceinline__ void look_up(const Segment& g, int first, int (&pg)[2]) const {
    const int32_t* table = a.page_table + (size_t)g.seq * a.table_pages;
    const int mine = steps(g);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int t = g.t0 + (4 * (first + lane) + wave) * 32 + 16 * h;
      pg[h] = first + lane < mine && t < g.to ? table[t >> a.page_shift] : -1;
    }
  }
  // asked for with the tokens themselves: the pages have to be there
  __device__ __forceinline__ void look_up_exponents(const Segment& g, int first, const int (&pg)[2]) {
    if constexpr (BLOCKS) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int t = g.t0 + (4 * (first + lane) + wave) * 32 + 16 * h;
        const size_t at = block_at((unsigned)pg[h] < (unsigned)a.n_pages ? pg[h] : 0, g.kvh, a.n_kv_heads, a.page_shift, t & ((1 << a.page_shift) - 1));
        exponents[h][0] = a.k_exponent[at];
        exponents[h][1] = a.v_exponent[at];
      }
    }
  }
  __device__ __forceinline__ float power(int h, int kv, int i) const { return power_of(exponent_of(__builtin_amdgcn_readlane(exponents[h][kv], i & 63))); }
  __device__ __forceinline__ void load_q(const Segment& g) {
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      q[c] = u32x4{0, 0, 0, 0};
      if (col < g.rows)
        q[c] = *reinterpret_cast<const u32x4*>(a.q + (size_t)(g.seq0 + col / group) * a.ld_q + (size_t)(g.kvh * group + col % group) * D + dim_of<D, SRC>(c, quad));
    }
  }
  __device__ __forceinline__ size_t row_of(const Segment& g, int t, int page) const {   // first element of token t's row
    return ((((size_t)((unsigned)page < (unsigned)a.n_pages ? page : 0) * a.n_kv_heads + g.kvh) << a.page_shift) + (t & ((1 << a.page_shift) - 1))) * D;
  }
  __device__ __forceinline__ void request_k(const Segment& g, int i, const int (&pg)[2], int (&next)[2]) {
    const int t = g.t0 + (4 * i + wave) * 32;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      next[h] = __builtin_amdgcn_readlane(pg[h], i & 63);
      const size_t at = row_of(g, t + 16 * h, next[h]) + col * D;
#pragma unroll
      for (int c = 0; c < R::KC; ++c) {
        if constexpr (FP8) raw.k[h][c] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(a.k) + at + 64 * c + 16 * quad);
        else raw.k[h][c] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.k) + at + 32 * c + 8 * quad);
      }
    }
  }
  __device__ __forceinline__ void request_v(const Segment& g, int i, const int (&next)[2]) {
    const int t = g.t0 + (4 * i + wave) * 32;
    typedef uint32_t words __attribute__((ext_vector_type(R::VW)));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const size_t at = row_of(g, t + 16 * h, next[h]) + 4 * quad * D + VD * col;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const void* p = FP8 ? (const void*)(static_cast<const uint8_t*>(a.v) + at + e * D) : (const void*)(static_cast<const uint16_t*>(a.v) + at + e * D);
        if constexpr (R::VW == 1) raw.v[4 * h + e][0] = *reinterpret_cast<const uint32_t*>(p);
        else {
          const words w = *reinterpret_cast<const words*>(p);
#pragma unroll
          for (int x = 0; x < R::VW; ++x) raw.v[4 * h + e][x] = w[x];
        }
      }
    }
  }
  __device__ __forceinline__ void start(const Segment& g) {   // a piece that nobody has asked for
    look_up(g, 0, pages);
    load_q(g);
    look_up_exponents(g, 0, pages);
    raw = R{};
    there[0] = there[1] = -1;
  }

  // The piece g, its first step asked for unless it is `fresh`; ahead: so is the first step of the piece `then` at the end.  Into o / ml_out, or
  // out where the piece is all that its rows see.  A fresh piece takes a step of nothing first, which asks for its first tokens: the code of
  // a step is then there before the loads of a whole chip are on their way, behind which it would be fetched (3 to 8 us).
  template <class SH>
  __device__ __forceinline__ void run(const Segment& g, bool fresh, bool ahead, const Segment& then, SH& sh, bool direct, float* o, float2* ml_out) {
  const float factor = a.scale * kLog2e * (SCALED ? a.k_scale[g.kvh] : 1.0f), scale = SCALED ? factor_of_scores(factor) : factor;
  if constexpr (SCALED) factor_to_query(q, factor);
  f32x4 acc[VD];
  float m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int j = 0; j < VD; ++j) acc[j] = f32x4{0, 0, 0, 0};
  const int mine = steps(g);
  int pages_then[2] = {-1, -1};
  if (ahead) look_up(then, 0, pages_then);
  ahead = ahead && steps(then) > 0;
  for (int i = fresh || mine == 0 ? -1 : 0; i < mine; ++i) {
    const int t = g.t0 + (4 * i + wave) * 32;
    const bool ok0 = (unsigned)there[0] < (unsigned)a.n_pages, ok1 = (unsigned)there[1] < (unsigned)a.n_pages;
    const bool whole = ok0 && ok1 && t >= g.from && t + 32 <= g.to;
    auto seen = [&](int h, int e) {                 // token e of the lane's four in half h
      const int tok = t + 16 * h + 4 * quad + e;
      return (h ? ok1 : ok0) && tok >= g.from && tok < g.to;
    };
    float power_k[2] = {1.0f, 1.0f}, power_v[2] = {1.0f, 1.0f};
    if constexpr (BLOCKS) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        power_k[h] = power(h, 0, i);
        power_v[h] = power(h, 1, i);
      }
    }
    u32x4 p;
    {
      f32x4 s[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
      for (int c = 0; c < KS; ++c) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          u32x4 kc;
          if constexpr (FP8) {
            const u32x2 x = widen4(raw.k[h][c / 2][2 * (c % 2)], power_k[h]), y = widen4(raw.k[h][c / 2][2 * (c % 2) + 1], power_k[h]);
            kc = u32x4{x[0], x[1], y[0], y[1]};
          } else kc = raw.k[h][c];
          s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kc), __builtin_bit_cast(bf16x8, q[c]), s[h], 0, 0, 0);
        }
      }
      if (!whole) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!seen(h, e)) s[h][e] = -INFINITY;
      }
      float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]))) * scale;
      if (__any(top > m)) {
        top = fmaxf(top, other_row16(top));
        top = fmaxf(top, other_half(top));
        const float raised = fmaxf(m, top + kSlack);
        const float shrink = exp2_fast(m - (raised == -INFINITY ? 0.0f : raised));
        l *= shrink;
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[j] *= shrink;
        m = raised;
      }
      const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        p[x] = pack2(exp2_fast(s[x / 2][2 * (x % 2)] * scale - from), exp2_fast(s[x / 2][2 * (x % 2) + 1] * scale - from));
        l = add_pair(p[x], l);          // the sum of what is multiplied with V
      }
    }
    int next[2] = {-1, -1};
    const bool more = i + 1 < mine;
    if (more) {
      if (((i + 1) & 63) == 0 && i > 0) {
        look_up(g, i + 1, pages);
        look_up_exponents(g, i + 1, pages);
      }
      request_k(g, i + 1, pages, next);
    } else if (ahead) {
      look_up_exponents(then, 0, pages_then);
      request_k(then, 0, pages_then, next);
    }
    if (!whole) {                                   // what no row sees must not turn a weight of 0 into NaN
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int x = 0; x < R::VW; ++x)
          if (!seen(e / 4, e % 4)) raw.v[e][x] = 0;
    }
#pragma unroll
    for (int jw = 0; jw < VD / 2; ++jw) {           // dimensions VD m + 2 jw and + 1
      uint32_t pair[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (FP8) pair[e] = widen4(raw.v[e][jw / 2], power_v[e / 4])[jw % 2];
        else pair[e] = raw.v[e][jw];
      }
#pragma unroll
      for (int odd = 0; odd < 2; ++odd) {
        u32x4 v;
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] = __builtin_amdgcn_perm(pair[2 * x + 1], pair[2 * x], odd ? 0x07060302u : 0x05040100u);
        acc[2 * jw + odd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, p), acc[2 * jw + odd], 0, 0, 0);
      }
    }
    if (more) request_v(g, i + 1, next);
    else if (ahead) request_v(then, 0, next);
    there[0] = next[0];
    there[1] = next[1];
  }
  if (ahead) load_q(then);
  pages[0] = pages_then[0];
  pages[1] = pages_then[1];

  // ---- the four wavefronts' results on one bound, added in their order
  __syncthreads();                                  // the last piece's reads of LDS are over
  l += other_row16(l);
  l += other_half(l);
  if (lane < 16) sh.ml[wave][lane] = make_float2(m, l);
  __syncthreads();
  {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sh.ml[w][col].x);
    const float shrink = exp2_fast(m - (top == -INFINITY ? 0.0f : top));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float* to = &sh.merge[wave][col][VD * (4 * quad + i)];
#pragma unroll
      for (int j = 0; j < VD; j += 4)
        *reinterpret_cast<f32x4*>(to + j) = f32x4{acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]} * shrink;
    }
    __syncthreads();
    const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * VD;
    if (row < g.rows) {
      float lr = 0.0f, mr = -INFINITY, x[VD];
#pragma unroll
      for (int w = 0; w < 4; ++w) mr = fmaxf(mr, sh.ml[w][row].x);
#pragma unroll
      for (int w = 0; w < 4; ++w) lr += sh.ml[w][row].y * exp2_fast(sh.ml[w][row].x - (mr == -INFINITY ? 0.0f : mr));
#pragma unroll
      for (int j = 0; j < VD; ++j) x[j] = sh.merge[0][row][d0 + j] + sh.merge[1][row][d0 + j] + sh.merge[2][row][d0 + j] + sh.merge[3][row][d0 + j];
      if (direct) {
        const float inv = lr == 0.0f ? 0.0f : (SCALED ? a.v_scale[g.kvh] : 1.0f) / lr;
        uint16_t* dst = a.out + (size_t)(g.seq0 + row / group) * a.ld_out + (size_t)(g.kvh * group + row % group) * D + d0;
#pragma unroll
        for (int j = 0; j < VD; j += 4)
          *reinterpret_cast<u32x2*>(dst + j) = u32x2{pack2(x[j] * inv, x[j + 1] * inv), pack2(x[j + 2] * inv, x[j + 3] * inv)};
      } else {
#pragma unroll
        for (int j = 0; j < VD; j += 4) *reinterpret_cast<f32x4*>(o + (size_t)row * D + d0 + j) = f32x4{x[j], x[j + 1], x[j + 2], x[j + 3]};
        if (d0 == 0) ml_out[row] = make_float2(mr, lr);
      }
    }
  }
  }
};

// The same for up to 128 rows: 32 per wavefront.
template <int D, int SRC>
__device__ __forceinline__ void run_many(const DecodeArgs& a, int group, const Segment& g, Shared<D, true>& sh, bool direct, float* o, float2* ml_out) {
  constexpr int KS = D / 16, DT = D / 32;
  constexpr bool SCALED = SRC == KV_PAGED_E4M3;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, row = kWaveRows * wave + (lane & 31);
  const int kvh = g.kvh;
  Stage<D, SRC> stage(sh.tiles);
  stage.k = static_cast<const char*>(a.k);
  stage.v = static_cast<const char*>(a.v);
  stage.exponents[0] = a.k_exponent;
  stage.exponents[1] = a.v_exponent;
  stage.kvh = kvh;
  stage.from = g.from;
  stage.to = g.t1;
  stage.table = a.page_table + (size_t)g.seq * a.table_pages;
  stage.page_shift = a.page_shift;
  stage.n_pages = a.n_pages;
  stage.n_kv_heads = a.n_kv_heads;
  TileRows<D> w;
  const int there = min(row, g.rows - 1);
  const uint16_t* src = a.q + (size_t)(g.seq0 + there / group) * a.ld_q + (size_t)(kvh * group + there % group) * D + 8 * half;
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) w.q[0][ks] = *reinterpret_cast<const bf16x8*>(src + 16 * ks);
  const float factor = a.scale * kLog2e * (SCALED ? a.k_scale[kvh] : 1.0f);
  if constexpr (SCALED) factor_to_query(w.q[0], factor);
  w.m[0] = -INFINITY;
  w.l[0] = 0.0f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) w.acc[0][dt] = f32x16{};
  const int last[NB] = {0x7fffffff}, first = g.t0 / kTile, n = (g.t1 - g.t0 + kTile - 1) / kTile;
  __syncthreads();                                  // the last piece's reads of LDS are over
  attend_tiles<D, SRC>(w, stage, first, kWaveRows * wave < g.rows ? n : 0, n, 0x7fffffff, last, SCALED ? factor_of_scores(factor) : factor);
  const float l = w.l[0] + other_half(w.l[0]);
  if (row >= g.rows) return;
  if (direct) {
    const float inv = l == 0.0f ? 0.0f : (SCALED ? a.v_scale[kvh] : 1.0f) / l;
    uint16_t* dst = a.out + (size_t)(g.seq0 + row / group) * a.ld_out + (size_t)(kvh * group + row % group) * D + 4 * half;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u32x2*>(dst + 32 * dt + 8 * i) = u32x2{pack2(w.acc[0][dt][4 * i] * inv, w.acc[0][dt][4 * i + 1] * inv), pack2(w.acc[0][dt][4 * i + 2] * inv, w.acc[0][dt][4 * i + 3] * inv)};
  } else {
    if (half == 0) ml_out[row] = make_float2(w.m[0], l);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(o + (size_t)row * D + 32 * dt + 8 * i + 4 * half) = f32x4{w.acc[0][dt][4 * i], w.acc[0][dt][4 * i + 1], w.acc[0][dt][4 * i + 2], w.acc[0][dt][4 * i + 3]};
  }
}

// MANY: prefixes are shared, or more than 16 query heads a key / value head: both bodies are there, also where no pass has more than 16 rows.  WHOLE: workgroup i does sequence i % n_seqs alone, and there is nothing to join.
template <int D, int SRC, bool MANY, bool WHOLE>
__global__ __launch_bounds__(kThreads, MANY ? 2 : 3) void k_attn_decode(DecodeCall c) {
  __shared__ __align__(16) Shared<D, MANY> sh;
  const DecodeArgs& a = c.a;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int n_groups = MANY ? a.n_groups : 0, n_items = n_groups + a.n_seqs;
  auto length = [&](int s) { return min(max(a.kv_len[s], 0), a.capacity); };
  auto units = [](int from, int to) { return to > from ? (to - (from & ~63) + kUnit - 1) / kUnit : 0; };

  if constexpr (WHOLE) {
    Few<D, SRC> few(a, c.sh.group);
    const int s = blockIdx.x % a.n_seqs;
    const Segment g = {(int)blockIdx.x / a.n_seqs, s, s, c.sh.group, 0, uniform(length(s)), 0, uniform(length(s))};
    few.start(g);
    few.run(g, true, false, g, sh, true, nullptr, nullptr);
    return;
  }

  // ---- units of every item, groups first
  for (int s = threadIdx.x; s < a.n_seqs; s += kThreads) sh.cum[n_groups + s] = units(0, length(s));
  __syncthreads();
  for (int g = wave; g < n_groups; g += 4) {
    const int first = a.first[g], behind = a.behind[g], prefix = a.prefix[g];
    int count = 0, src = -1;
    for (int s0 = first; s0 < behind; s0 += 64) {
      const uint64_t who = __ballot(s0 + lane < behind && length(min(s0 + lane, a.n_seqs - 1)) >= prefix);
      if (src < 0 && who) src = s0 + __builtin_ctzll(who);
      count += __popcll(who);
    }
    const bool active = count >= 2;
    if (active)
      for (int s = first + lane; s < behind; s += 64)
        if (length(s) >= prefix) sh.cum[n_groups + s] = units(prefix, length(s));
    if (lane == 0) {
      sh.group_src[g] = active ? src : -1;
      sh.cum[g] = active ? (prefix + kUnit - 1) / kUnit * ((behind - first + c.sh.per_pass - 1) / c.sh.per_pass) : 0;
    }
  }
  __syncthreads();
  // lane g: the sequences and the prefix of group g, if it shares
  int my_first = 0, my_behind = 0, my_prefix = 0;
  if (lane < n_groups && sh.group_src[lane] >= 0) {
    my_first = a.first[lane];
    my_behind = a.behind[lane];
    my_prefix = a.prefix[lane];
  }
  auto shared_by = [&](int s, int len) {            // the prefix that a sequence (the same in all lanes) shares with others
    const uint64_t who = __ballot(my_first <= s && s < my_behind && len >= my_prefix);
    return who ? __builtin_amdgcn_readlane(my_prefix, __builtin_ctzll(who)) : 0;
  };
  // ---- exclusive sums, in place
  {
    const int per = (n_items + kThreads - 1) / kThreads, lo = min((int)threadIdx.x * per, n_items), hi = min(lo + per, n_items);
    int sum = 0;
    for (int i = lo; i < hi; ++i) sum += sh.cum[i];
    const int run = wave_scan(sum);
    if (lane == 63) sh.part[wave] = run;
    __syncthreads();
    int at = run - sum;
    for (int w = 0; w < wave; ++w) at += sh.part[w];
    for (int i = lo; i < hi; ++i) {
      const int v = sh.cum[i];
      sh.cum[i] = at;
      at += v;
    }
    if (threadIdx.x == kThreads - 1) sh.cum[n_items] = sh.part[0] + sh.part[1] + sh.part[2] + sh.part[3];
    __syncthreads();
  }
  const int per_head = uniform(sh.cum[n_items]), all = per_head * a.n_kv_heads;
  const int chunk = max((all + (int)gridDim.x - 1) / (int)gridDim.x, 1);

  const Layout y = layout(a.n_seqs, a.n_kv_heads, c.sh.group, c.sh.n_passes, D);
  char* ws = static_cast<char*>(a.ws);

  // ---- this workgroup's chunk, piece by piece
  const int begin = (int)min((int64_t)blockIdx.x * chunk, (int64_t)all), end = min(begin + chunk, all);
  struct Piece {
    Segment g;
    int units;
    bool direct;
    float* o;
    float2* ml;
  };
  auto piece_at = [&](int u) {
    Piece p;
    Segment& g = p.g;
    const int h = u / per_head, in_head = u % per_head;
    int lo = 0, hi = n_items - 1;                   // last item that begins at or before the unit (those of no units come before it)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (sh.cum[mid] <= in_head) lo = mid; else hi = mid - 1;
    }
    const int it = uniform(lo), first = uniform(sh.cum[it]), n = uniform(sh.cum[it + 1]) - first;
    int from_unit = in_head - first, to_unit = min(from_unit + end - u, n);
    g.kvh = h;
    p.direct = false;
    if (it < n_groups) {
      const int tiles = (a.prefix[it] + kUnit - 1) / kUnit, pass = from_unit / tiles;
      from_unit -= pass * tiles;
      to_unit = min(to_unit - pass * tiles, tiles);
      g.seq = uniform(sh.group_src[it]);
      g.seq0 = a.first[it] + pass * c.sh.per_pass;
      g.rows = min(c.sh.per_pass, a.behind[it] - g.seq0) * c.sh.group;
      g.from = 0;
      g.to = a.prefix[it];
      g.t0 = from_unit * kUnit;
      g.t1 = min(to_unit * kUnit, g.to);
      const size_t slot = (size_t)blockIdx.x + h * c.sh.n_passes + c.pass_base[it] + pass;
      p.o = reinterpret_cast<float*>(ws + y.prefix_o) + slot * kRowsPass * D;
      p.ml = reinterpret_cast<float2*>(ws + y.prefix_ml) + slot * kRowsPass;
    } else {
      const int s = it - n_groups;
      g.seq = g.seq0 = s;
      g.rows = c.sh.group;
      g.to = uniform(length(s));
      g.from = shared_by(s, g.to);
      const size_t slot = (size_t)blockIdx.x + (size_t)h * a.n_seqs + s;
      p.direct = g.from == 0 && from_unit == 0 && to_unit == n;
      p.o = reinterpret_cast<float*>(ws + y.own_o) + slot * c.sh.group * D;
      p.ml = reinterpret_cast<float2*>(ws + y.own_ml) + slot * c.sh.group;
      g.t0 = (g.from & ~63) + from_unit * kUnit;
      g.t1 = min((g.from & ~63) + to_unit * kUnit, g.to);
    }
    g.t0 = uniform(g.t0);
    g.t1 = uniform(g.t1);
    g.rows = uniform(g.rows);
    p.units = uniform(to_unit - from_unit);
    return p;
  };
  // first the pieces of many rows, then the others: in one loop both bodies would keep registers for each other
  if constexpr (MANY) {
    for (int u = begin; u < end;) {
      const Piece p = piece_at(u);
      u += p.units;
      if (p.g.rows > kFewRows) run_many<D, SRC>(a, c.sh.group, p.g, sh, p.direct, p.o, p.ml);
    }
    asm volatile("" ::: "memory");
  }
  int u = begin;
  auto next_few = [&](Piece& p) {
    while (u < end) {
      p = piece_at(u);
      u += p.units;
      if (!MANY || p.g.rows <= kFewRows) return true;
    }
    return false;
  };
  Piece p, then;
  Few<D, SRC> few(a, c.sh.group);
  for (int round = 0;; ++round) {
    const bool more = next_few(then);               // while the first tokens of piece p are on their way
    if (round) few.run(p.g, round == 1, more, then.g, sh, p.direct, p.o, p.ml);
    else if (more) few.start(then.g);
    if (!more) break;
    p = then;
  }

  // ---- where the join finds every row's pieces
  Meta* meta = reinterpret_cast<Meta*>(ws + y.meta);
  for (int i = blockIdx.x * kThreads + threadIdx.x; i < a.n_kv_heads * a.n_seqs; i += gridDim.x * kThreads) {
    const int h = i / a.n_seqs, s = i % a.n_seqs, it = n_groups + s;
    Meta w = make_int4(0, 0, 0, 0);
    for (int g = 0; g < n_groups; ++g) {
      if (s < a.first[g] || s >= a.behind[g]) continue;
      if (sh.group_src[g] >= 0 && length(s) >= a.prefix[g]) {
        const int n = (a.prefix[g] + kUnit - 1) / kUnit, pass = (s - a.first[g]) / c.sh.per_pass;
        const int u0 = h * per_head + sh.cum[g] + pass * n, w0 = u0 / chunk, w1 = (u0 + n - 1) / chunk;
        w.z = w0 + h * c.sh.n_passes + c.pass_base[g] + pass;
        w.w = (w1 - w0 + 1) | ((s - a.first[g]) % c.sh.per_pass * c.sh.group) << 16;
      }
      break;
    }
    const int u0 = h * per_head + sh.cum[it], n = sh.cum[it + 1] - sh.cum[it];
    if (n > 0) {
      const int w0 = u0 / chunk, w1 = (u0 + n - 1) / chunk;
      w.x = w0 + i;
      w.y = w0 == w1 && w.w == 0 ? -1 : w1 - w0 + 1;
    }
    meta[i] = w;
  }
}

// One wavefront (W = 4: four, sharing out the pieces) per query row: the pieces of its prefix and its own, on one bound.
template <int D, int W>
__global__ __launch_bounds__(kThreads) void k_join(DecodeCall c, bool scaled) {
  constexpr int E = D / 64;                          // dimensions per lane
  __shared__ float part[4][D];
  const DecodeArgs& a = c.a;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), group = c.sh.group;
  const int row = W == 4 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave;
  if (row >= a.n_seqs * a.n_heads) return;
  const int s = row / a.n_heads, head = row % a.n_heads, h = head / group, r = head % group;
  const Layout y = layout(a.n_seqs, a.n_kv_heads, group, c.sh.n_passes, D);
  const char* ws = static_cast<const char*>(a.ws);
  const Meta w = reinterpret_cast<const Meta*>(ws + y.meta)[h * a.n_seqs + s];
  if (w.y < 0) return;
  const int n_pre = w.w & 0xffff, n = n_pre + w.y;
  const float* pre_o = reinterpret_cast<const float*>(ws + y.prefix_o) + ((size_t)w.z * kRowsPass + (w.w >> 16) + r) * D;
  const float2* pre_ml = reinterpret_cast<const float2*>(ws + y.prefix_ml) + (size_t)w.z * kRowsPass + (w.w >> 16) + r;
  const float* own_o = reinterpret_cast<const float*>(ws + y.own_o) + ((size_t)w.x * group + r) * D;
  const float2* own_ml = reinterpret_cast<const float2*>(ws + y.own_ml) + (size_t)w.x * group + r;
  float m = -INFINITY, l = 0.0f, x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = 0.0f;
  // up to 64 pieces at a time: lane i weighs piece i; a wavefront adds up every W-th, kBatch of them on their way at a time
  constexpr int kBatch = 8;
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int i = i0 + lane, count = min(64, n - i0);
    float2 ml = make_float2(-INFINITY, 0.0f);
    if (i < n) ml = i < n_pre ? pre_ml[(size_t)i * kRowsPass] : own_ml[(size_t)(i - n_pre) * group];
    float top = ml.x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float raised = fmaxf(m, top), to = raised == -INFINITY ? 0.0f : raised, shrink = exp2_fast(m - to);
    const float weight = exp2_fast(ml.x - to);
    float sum = ml.y * weight;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
    l = l * shrink + sum;
    m = raised;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= shrink;
    for (int k0 = W == 4 ? wave : 0; k0 < count; k0 += W * kBatch) {
      float v[kBatch][E], f[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int k = min(k0 + W * b, count - 1), p = i0 + k;
        f[b] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), k));
        const float* o = p < n_pre ? pre_o + (size_t)p * kRowsPass * D : own_o + (size_t)(p - n_pre) * group * D;
#pragma unroll
        for (int e = 0; e < E; ++e) v[b][e] = o[E * lane + e];
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b)            // behind the last piece it is read again, and left out: its values may be infinite
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = k0 + W * b < count ? fmaf(f[b], v[b][e], x[e]) : x[e];
    }
  }
  if constexpr (W == 4) {                            // all four have the same bound and sum
#pragma unroll
    for (int e = 0; e < E; ++e) part[wave][E * lane + e] = x[e];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = part[0][E * lane + e] + part[1][E * lane + e] + part[2][E * lane + e] + part[3][E * lane + e];
  }
  const float inv = l == 0.0f ? 0.0f : (scaled ? a.v_scale[h] : 1.0f) / l;
  uint16_t* dst = a.out + (size_t)s * a.ld_out + (size_t)head * D + E * lane;
  if constexpr (E == 2) *reinterpret_cast<uint32_t*>(dst) = pack2(x[0] * inv, x[1] * inv);
  else *dst = (uint16_t)pack2(x[0] * inv, 0.0f);
}

template <int D, int SRC>
hipError_t launch(const DecodeCall& c, hipStream_t s) {
  const bool many = c.sh.group > kFewRows || c.a.n_groups > 0;
  if (!many && c.a.capacity <= kWholeTokens) {
    k_attn_decode<D, SRC, false, true><<<(unsigned)(c.a.n_kv_heads * c.a.n_seqs), kThreads, 0, s>>>(c);
    return hipGetLastError();
  }
  // never more workgroups than units there can be
  const int64_t most = (int64_t)c.a.n_kv_heads * (c.a.n_seqs + c.sh.n_passes) * ((c.a.capacity + kUnit - 1) / kUnit + 1);
  const unsigned grid = (unsigned)std::min<int64_t>(many ? kWorkgroups : kWorkgroupsFew, most);
  if (many) k_attn_decode<D, SRC, true, false><<<grid, kThreads, 0, s>>>(c);
  else k_attn_decode<D, SRC, false, false><<<grid, kThreads, 0, s>>>(c);
  if (hipError_t e = hipGetLastError()) return e;
  const int rows = c.a.n_seqs * c.a.n_heads;
  if (rows <= 1024) k_join<D, 4><<<rows, kThreads, 0, s>>>(c, SRC == KV_PAGED_E4M3);
  else k_join<D, 1><<<(rows + 3) / 4, kThreads, 0, s>>>(c, SRC == KV_PAGED_E4M3);
  return hipGetLastError();
}
template <int D>
hipError_t launch_of(const DecodeCall& c, int source, hipStream_t s) {
  return source == KV_PAGED ? launch<D, KV_PAGED>(c, s) : source == KV_PAGED_E4M3 ? launch<D, KV_PAGED_E4M3>(c, s) : launch<D, KV_PAGED_BLOCKS>(c, s);
}

}  // namespace

size_t attn_decode_workspace_bytes(int n_seqs, int n_heads, int n_kv_heads, int head_dim) {
  const int group = n_heads / n_kv_heads, per_pass = kRowsPass / group;
  // passes of any way to share: a group has two sequences or more
  const int most = n_seqs < 2 ? 0 : n_seqs / per_pass + std::min(MES_MAX_EXPERTS, n_seqs / 2);
  return layout(n_seqs, n_kv_heads, group, most, head_dim).total;
}

hipError_t launch_attn_decode(const DecodeArgs& a, int source, hipStream_t s) {
  DecodeCall c;
  c.a = a;
  c.sh.group = a.n_heads / a.n_kv_heads;
  c.sh.per_pass = kRowsPass / c.sh.group;
  c.sh.n_passes = 0;
  for (int g = 0; g < a.n_groups; ++g) {
    c.pass_base[g] = c.sh.n_passes;
    c.sh.n_passes += (a.behind[g] - a.first[g] + c.sh.per_pass - 1) / c.sh.per_pass;
  }
  return a.head_dim == 128 ? launch_of<128>(c, source, s) : launch_of<64>(c, source, s);
}

}  // namespace mes
