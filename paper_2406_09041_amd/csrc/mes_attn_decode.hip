// One token of every sequence against the paged cache, prefixes that an expert's sequences share read once.  Bound by HBM:
// every distinct cached token is read once, 2 head_dim values per key / value head, for 4 head_dim n_heads operations.
//
// Work is a flat line of costs.  First, per key / value head, what many query rows read together: passes of up to 128 rows over a shared
// prefix, in tiles of 64 tokens, which a workgroup's four wavefronts do together.  Then what every sequence has of its own, in steps of 32 tokens,
// which a wavefront does alone and waits for nobody (in teams of four with their sums added up in LDS, sequences of 16 to 4096 tokens
// took 104 us instead of 91, as beginning and ending a piece cost 4 us each).  The line is cut into equal chunks, wherever that falls: all wavefronts are
// equally busy however the lengths are spread, and the launch does not depend on the lengths, which stay on
// the device (every workgroup adds them up for itself).  Where there are few sequences and heads, they are cut in equal parts instead (few_items).  A piece of the line that does not cover a sequence alone leaves (bound, sum,
// weighted values) in the workspace, and k_join adds the pieces of a row in their order.
//
// A sequence's own tokens, up to 16 heads per key / value head: a wavefront takes 32 tokens at a time.  Scores are formed transposed,
// S^T = K Q^T with v_mfma_f32_16x16x32_bf16: K's operand is 16 tokens x 8 dimensions per lane straight from memory, and the result
// holds one query row (lane & 15) and tokens 4 g + (0..3) per lane (g = lane / 16), which rounded to bf16 IS the operand P^T of
// O^T = V^T P^T over the 32 tokens in the order (4 g + i, 16 + 4 g + i).  V is read by rows, 16 lanes a row, lane r the dimensions
// VD r .. VD r + VD - 1 of its 8 tokens: product j of VD then yields the dimensions VD m + j, and its operand
// is pairs of 16-bit halves put together, one v_perm each.  So neither keys nor values pass through LDS.  Of the 16 columns of a
// tile 4 (n_heads / n_kv_heads) are used where nothing is shared: the matrix cores are idle most of the time anyway.
//
// Prefixes: up to 128 rows share keys and values in LDS (mes_attn_tiles.h), bound by the matrix cores from about 100 rows on; also those of a
// sequence alone where more than 16 query heads share a key / value head.  Passes of up to 16 rows stream their tokens as above where that pays
// (streaming_pays).
//
// Weights are rounded to bf16 for the product with V, as the matrix cores take both operands alike, and summed as rounded: they still add up
// to 1, and a row's error grows by at most 2^-8 of its weighted values' size (measured against 64 bits: 0.0020 of the rows' norm, 0.0017
// with weights in fp32).
//
// Measured (head_dim 128, 32 heads over 8 key / value heads): 256 sequences of 0 to 8192 tokens 160 us, 5.0 TB/s of the 5.96 that a
// pass that only reads reaches; the same over e4m3 codes 91 us, 4.4 TB/s (the wavefronts end within 81 us, half of them within 74, and the join
// takes 7); 256 of 735 tokens over blocks 76 us, 5.1 TB/s; 256 of 9 experts with prompts of 64 to 4000 tokens over blocks 109 us; 64 of 16 experts with
// prompts of 512 to 1600 tokens 33 to 36 us; 96 behind 8200 shared tokens of an e4m3 cache 50 us, of which 10 us are products at the library's
// rate; one sequence of 200 tokens 8.3 us, of 8000 12.4.  Two steps of a wavefront on their way instead of one: no faster over codes, and spilled over bf16; the heads
// of a sequence one behind the other on the line, instead of the sequences of a head: the same.
#include "mes_attn_tiles.h"

namespace mes {
namespace {

constexpr bool has_codes(int source) { return source != KV_PAGED; }

constexpr int kThreads = 256, kWaves = kThreads / 64, kStep = 32, kRowsPass = 128, kFewRows = 16;
// Costs on the line, in steps of a wavefront: of a tile of the larger body, of beginning and ending what a pass or a sequence does there, and
// the same of a sequence's own part in the smaller one.  Under load, heads of 128: a step takes 2.7 us over codes and 5.4 over bf16, a piece 5 us more, a workgroup's
// tile 2.3 to 2.6 us over codes and 3.1 over bf16 (four wavefronts' time).  Tiles and passes are set higher than that: they come first on the line, and what is late there
// ends last (256 sequences of 9 experts over blocks: 162 us with tiles at 3 and passes at nothing, 109 with these).
template <int SRC>
struct Cost {
  static constexpr uint32_t kTile = has_codes(SRC) ? 7 : 4, kBegin = has_codes(SRC) ? 12 : 7, kOwn = has_codes(SRC) ? 3 : 2;
  static constexpr uint32_t kTileStreamed = 64 / kStep, kBeginStreamed = kWaves * kOwn;   // of a pass whose tokens are streamed
};
// Costs of a sequence and head never pass kMostCosts (u + 2), u = capacity / 128 (4 u + 4 steps, 2 u + 2 tiles at most), so that those of a call, and what they
// are rounded up by, fit 32 bits (see decode_fits).  Sequences that share pay for the tokens behind the prefix, those shorter than it for their own alone, and there are
// passes for half as many as both at most, but for groups of an odd number in passes of two, one more, of which the two that share pay for.
// Narrow: the own part and half a pass; wide: the same, from tiles.  What is rounded up: a 512th, which narrow groups have room for; wide ones are not.
template <int SRC>
constexpr bool costs_fit() {
  typedef Cost<SRC> C;
  return 4 + C::kTile < kMostCosts && C::kOwn + 5 + (C::kBegin + 2 * C::kTile + 1) / 2 < 2 * kMostCosts &&   // 4 u + 5 steps, 2 u + 2 tiles
         3 * kWaves <= kMostCosts && 6 * kWaves <= 2 * kMostCosts;                                            // (2 u + 2 tiles and a beginning) 3 / 2
}
static_assert(costs_fit<KV_PAGED>() && costs_fit<KV_PAGED_E4M3>() && costs_fit<KV_PAGED_BLOCKS>(), "work numbers of 32 bits");
// Workgroups of a launch: two per compute unit, which is what the chip holds with the larger body; without it three fit, and were as fast
// or slower (256 sequences of 735 tokens 92 us instead of 76).
constexpr int kWorkgroups = 512;
// Up to this many tokens a sequence is one workgroup's, where nothing is shared: no second launch to add up pieces (one
// sequence of 200 tokens, when it was made: 9.2 us, 12.4 with it).
constexpr int kWholeTokens = 512;
// Few sequences and heads are not put on the line: with up to a wavefront's work each, a row's pieces are so many that adding them up takes longer than
// they do (one sequence of 60000 tokens, 8 heads over one key / value head: 52 us, 20 as in few_items; of 8000, 32 over 8: 18.0 and 12.4; 32
// of 700, 28 over 4: 19.4 and 15.5).  From about 200 items on the line is as fast or faster, and where a part would be longer than
// kMostUnits, as parts of one length leave compute units idle (one of 60000, 40 heads of their own: 219 us and 256).
constexpr int kLeastStreamed = 256;   // tokens
constexpr int kFewItems = 192, kFewSeqs = 256, kMostUnits = 8;
static_assert(kFewItems <= kWorkgroups && kFewSeqs >= kFewItems && kFewSeqs % 64 == 0, "an item has a workgroup, a lane as many sequences as another");
static_assert(kThreads == kTileThreads && kRowsPass == kTileWaves * kWaveRows, "the workgroups of both bodies are the same");

struct Shape {                       // what host and device derive alike
  int group, per_pass, n_passes;     // query heads per key / value head, sequences per pass, passes of all groups
};

// Of the workspace: partial results [slot][rows][D] floats and [slot][rows] (bound, sum), of passes and of sequences' own parts.
struct Layout {
  size_t prefix_o, prefix_ml, own_o, own_ml, meta, total;
};

__host__ __device__ inline Layout layout(int n_seqs, int n_kv_heads, int group, int n_passes, int head_dim) {
  const size_t pre = (size_t)(n_passes ? kWorkgroups + n_kv_heads * n_passes : 0) * kRowsPass;
  const size_t own = (size_t)((group > kFewRows ? 1 : kWaves) * kWorkgroups + n_kv_heads * n_seqs) * group;
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

template <int D, int SRC>
struct Raw {                                        // 32 tokens of keys and values on their way, as the loads bring them
  static constexpr bool FP8 = has_codes(SRC);
  static constexpr int VD = D / 16, KC = FP8 ? D / 64 : D / 32, VW = VD * (FP8 ? 1 : 2) / 4;
  typedef uint32_t Words __attribute__((ext_vector_type(VW)));
  u32x4 k[2][KC];
  Words v[8];
};

// first dimension of the 8 that a lane holds in product c of K Q^T
template <int D, int SRC>
__device__ __forceinline__ int dim_of(int c, int g) {
  return has_codes(SRC) ? 64 * (c / 2) + 16 * g + 8 * (c % 2) : 32 * c + 8 * g;
}

struct Segment {                                    // a piece of the line
  int kvh, seq, seq0, rows;                         // key / value head; page table; sequence of row 0; query rows
  int from, to, t0, t1;                             // tokens of [from, to) in [t0, t1), t0 a multiple of a tile or a step
};

template <int D>
struct Merge {                                      // a workgroup's four wavefronts of one piece
  float o[4][kFewRows][D + 4];
  float2 ml[4][kFewRows];
};
struct Nothing {};
// What a decode kernel is made for: the line of sequences' own parts alone; few items before it; prefixes that are shared, or more than 16 query heads a key /
// value head; prefixes of few rows.  What a call does not need costs its kernel registers, so each has its own (few_items beside the line: up to 3%,
// passes that are streamed beside those that are not: 5%).
enum Mode { LINE, FEW_ITEMS, MANY_ROWS, STREAMED };
template <int D, int MODE>
struct Shared {
  [[no_unique_address]] std::conditional_t<(MODE >= MANY_ROWS), TileLds<D>, Nothing> tiles;
  [[no_unique_address]] std::conditional_t<MODE == FEW_ITEMS, Merge<D>, Nothing> merge;
  uint32_t cum[MES_MAX_SEQS + MES_MAX_EXPERTS + 1];
  int group_src[MES_MAX_EXPERTS];                   // first sequence as long as the prefix, -1: fewer than two are
  uint32_t part[4];
};

// The weighted sum over a piece with up to 16 query rows.  Pieces follow one another without a pause: a wavefront asks for the next piece's
// first tokens where it would ask for more of this one's, and knows their pages by then.  TEAM: the workgroup's wavefronts take every fourth step
// of a piece and add up their results; else a piece is a wavefront's, which waits for nobody.
template <int D, int SRC, bool TEAM>
struct Few {
  static constexpr bool FP8 = has_codes(SRC), SCALED = SRC == KV_PAGED_E4M3, BLOCKS = SRC == KV_PAGED_BLOCKS;
  static constexpr int VD = D / 16, KS = D / 32, kBatch = 32;   // kBatch: steps whose pages are looked up together
  typedef Raw<D, SRC> R;
  const DecodeArgs& a;
  int group, lane, wave, col, quad;
  u32x4 q[KS];                                      // Q^T operands
  R raw;                                            // the step that comes next
  int there[2];                                     // its pages
  int pages;                                        // of the halves of kBatch steps of the piece, one half per lane
  int exponents[2];                                 // blocks: of keys and values on these pages

  __device__ Few(const DecodeArgs& args, int g) : a(args), group(g), lane(threadIdx.x & 63), wave(uniform(threadIdx.x >> 6)), col(lane & 15), quad(lane >> 4) {}

  __device__ __forceinline__ int token_of(const Segment& g, int step) const { return g.t0 + (TEAM ? 4 * step + wave : step) * kStep; }
  __device__ __forceinline__ int steps(const Segment& g) const {
    const int all = (g.t1 - g.t0 + kStep - 1) / kStep;
    return TEAM ? (all - wave + 3) / 4 : all;
  }
  // the pages of steps first .. first + kBatch - 1
  __device__ __forceinline__ int look_up(const Segment& g, int first) const {
    const int t = token_of(g, first + lane / 2) + lane % 2 * 16;
    return t < g.t1 ? (a.page_table + (size_t)g.seq * a.table_pages)[t >> a.page_shift] : -1;
  }
  // asked for with the tokens themselves: the pages have to be there
  __device__ __forceinline__ void look_up_exponents(const Segment& g, int first, int pg) {
    if constexpr (BLOCKS) {
      const int t = token_of(g, first + lane / 2) + lane % 2 * 16;
      const size_t at = block_at((unsigned)pg < (unsigned)a.n_pages ? pg : 0, g.kvh, a.n_kv_heads, a.page_shift, t & ((1 << a.page_shift) - 1));
      exponents[0] = a.k_exponent[at];
      exponents[1] = a.v_exponent[at];
    }
  }
  __device__ __forceinline__ static int lane_of(int step, int half) { return (step & (kBatch - 1)) * 2 + half; }
  __device__ __forceinline__ float power(int h, int kv, int i) const { return power_of(exponent_of(__builtin_amdgcn_readlane(exponents[kv], lane_of(i, h)))); }
  __device__ __forceinline__ void load_q(const Segment& g, u32x4 (&to)[KS]) const {
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      to[c] = u32x4{0, 0, 0, 0};
      if (col < g.rows)
        to[c] = *reinterpret_cast<const u32x4*>(a.q + (size_t)(g.seq0 + col / group) * a.ld_q + (size_t)(g.kvh * group + col % group) * D + dim_of<D, SRC>(c, quad));
    }
  }
  __device__ __forceinline__ size_t row_of(const Segment& g, int t, int page) const {   // first element of token t's row
    return ((((size_t)((unsigned)page < (unsigned)a.n_pages ? page : 0) * a.n_kv_heads + g.kvh) << a.page_shift) + (t & ((1 << a.page_shift) - 1))) * D;
  }
  // The rows of 16 tokens are at a base that all lanes share, a lane's bytes at a distance that all of them share.
  __device__ __forceinline__ void request_k(const Segment& g, int i, int pg, int (&next)[2]) {
    constexpr int kItem = FP8 ? 1 : 2;
    const uint32_t mine = col * D * kItem + 16 * quad;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      next[h] = __builtin_amdgcn_readlane(pg, lane_of(i, h));
      const char* base = static_cast<const char*>(a.k) + row_of(g, token_of(g, i) + 16 * h, next[h]) * kItem;
#pragma unroll
      for (int c = 0; c < R::KC; ++c) raw.k[h][c] = *reinterpret_cast<const u32x4*>(base + (mine + 64 * c));
    }
  }
  __device__ __forceinline__ void request_v(const Segment& g, int i, const int (&next)[2]) {
    constexpr int kItem = FP8 ? 1 : 2;
    const uint32_t mine = (4 * quad * D + VD * col) * kItem;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char* base = static_cast<const char*>(a.v) + row_of(g, token_of(g, i) + 16 * h, next[h]) * kItem;
#pragma unroll
      for (int e = 0; e < 4; ++e) raw.v[4 * h + e] = *reinterpret_cast<const typename R::Words*>(base + (mine + e * D * kItem));
    }
  }
  __device__ __forceinline__ void start(const Segment& g) {   // a piece that nobody has asked for
    pages = look_up(g, 0);
    load_q(g, q);
    look_up_exponents(g, 0, pages);
    raw = R{};
    there[0] = there[1] = -1;
  }

  // The piece g, its first step asked for unless it is `fresh`; ahead: so is the first step of the piece `then` at the end.  Into o / ml_out, or
  // out where the piece is all that its rows see.  A fresh piece takes a step of nothing first, which asks for its first tokens: the code of
  // a step is then there before the loads of a whole chip are on their way, behind which it would be fetched (3 to 8 us).
  __device__ __forceinline__ void run(const Segment& g, bool fresh, bool ahead, const Segment& then, Merge<D>* sh, bool direct, float* o, float2* ml_out) {
  const float factor = a.scale * kLog2e * (SCALED ? a.k_scale[g.kvh] : 1.0f), scale = SCALED ? factor_of_scores(factor) : factor;
  if constexpr (SCALED) factor_to_query(q, factor);
  f32x4 acc[VD];
  float m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int j = 0; j < VD; ++j) acc[j] = f32x4{0, 0, 0, 0};
  const int mine = steps(g);
  int pages_then = -1, pages_next = -1;             // of the next piece, of this one's next batch
  u32x4 q_then[KS];                                 // asked for long before it is needed: a wavefront would wait for it between pieces
  if (ahead) {
    pages_then = look_up(then, 0);
    load_q(then, q_then);
  }
  const bool another = ahead;
  ahead = ahead && steps(then) > 0;
  for (int i = fresh || mine == 0 ? -1 : 0; i < mine; ++i) {
    const int t = token_of(g, i);
    const bool ok0 = (unsigned)there[0] < (unsigned)a.n_pages, ok1 = (unsigned)there[1] < (unsigned)a.n_pages;
    const bool whole = ok0 && ok1 && t >= g.from && t + kStep <= g.t1;
    auto seen = [&](int h, int e) {                 // token e of the lane's four in half h
      const int tok = t + 16 * h + 4 * quad + e;
      return (h ? ok1 : ok0) && tok >= g.from && tok < g.t1;
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
      if (((i + 1) & (kBatch - 1)) == 0 && i > 0) {
        pages = pages_next;
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
        if (!seen(e / 4, e % 4)) raw.v[e] = typename R::Words(0);
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
    if (more) {
      request_v(g, i + 1, next);
      if (((i + 2) & (kBatch - 1)) == 0) pages_next = look_up(g, i + 2);
    } else if (ahead) request_v(then, 0, next);
    there[0] = next[0];
    there[1] = next[1];
  }
  if (another) {
#pragma unroll
    for (int c = 0; c < KS; ++c) q[c] = q_then[c];
  }
  pages = pages_then;
  l += other_row16(l);
  l += other_half(l);
  if constexpr (!TEAM) {
    // lane (col, quad) has row col, dimensions VD (4 quad + i) ..
    if (col >= g.rows) return;
    const float inv = l == 0.0f ? 0.0f : (SCALED ? a.v_scale[g.kvh] : 1.0f) / l;
    uint16_t* dst = a.out + (size_t)(g.seq0 + col / group) * a.ld_out + (size_t)(g.kvh * group + col % group) * D;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < VD; j += 4) {
        const int d = VD * (4 * quad + i) + j;
        if (direct) *reinterpret_cast<u32x2*>(dst + d) = u32x2{pack2(acc[j][i] * inv, acc[j + 1][i] * inv), pack2(acc[j + 2][i] * inv, acc[j + 3][i] * inv)};
        else *reinterpret_cast<f32x4*>(o + (size_t)col * D + d) = f32x4{acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]};
      }
    if (!direct && quad == 0) ml_out[col] = make_float2(m, l);
    return;
  } else {

  // ---- the four wavefronts' results on one bound, added in their order
  if (lane < 16) sh->ml[wave][lane] = make_float2(m, l);
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, sh->ml[w][col].x);
  const float shrink = exp2_fast(m - (top == -INFINITY ? 0.0f : top));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float* to = &sh->o[wave][col][VD * (4 * quad + i)];
#pragma unroll
    for (int j = 0; j < VD; j += 4)
      *reinterpret_cast<f32x4*>(to + j) = f32x4{acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i]} * shrink;
  }
  __syncthreads();
  const int row = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * VD;
  if (row >= g.rows) return;
  float lr = 0.0f, mr = -INFINITY, x[VD];
#pragma unroll
  for (int w = 0; w < 4; ++w) mr = fmaxf(mr, sh->ml[w][row].x);
#pragma unroll
  for (int w = 0; w < 4; ++w) lr += sh->ml[w][row].y * exp2_fast(sh->ml[w][row].x - (mr == -INFINITY ? 0.0f : mr));
#pragma unroll
  for (int j = 0; j < VD; ++j) x[j] = sh->o[0][row][d0 + j] + sh->o[1][row][d0 + j] + sh->o[2][row][d0 + j] + sh->o[3][row][d0 + j];
  if (!direct) {
#pragma unroll
    for (int j = 0; j < VD; j += 4) *reinterpret_cast<f32x4*>(o + (size_t)row * D + d0 + j) = f32x4{x[j], x[j + 1], x[j + 2], x[j + 3]};
    if (d0 == 0) ml_out[row] = make_float2(mr, lr);
    return;
  }
  const float inv = lr == 0.0f ? 0.0f : (SCALED ? a.v_scale[g.kvh] : 1.0f) / lr;
  uint16_t* dst = a.out + (size_t)(g.seq0 + row / group) * a.ld_out + (size_t)(g.kvh * group + row % group) * D + d0;
#pragma unroll
  for (int j = 0; j < VD; j += 4)
    *reinterpret_cast<u32x2*>(dst + j) = u32x2{pack2(x[j] * inv, x[j + 1] * inv), pack2(x[j + 2] * inv, x[j + 3] * inv)};
  }
  }
};

// The same for up to 128 rows: 32 per wavefront.
template <int D, int SRC>
__device__ __forceinline__ void run_many(const DecodeArgs& a, int group, const Segment& g, TileLds<D>& tiles, bool direct, float* o, float2* ml_out) {
  constexpr int KS = D / 16, DT = D / 32;
  constexpr bool SCALED = SRC == KV_PAGED_E4M3;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, row = kWaveRows * wave + (lane & 31);
  const int kvh = g.kvh;
  Stage<D, SRC> stage(tiles);
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

// Sequences of up to kWholeTokens: workgroup i does sequence i % n_seqs alone, and there is nothing to join.
template <int D, int SRC>
__global__ __launch_bounds__(kThreads, 3) void k_attn_decode_whole(DecodeCall c) {
  __shared__ __align__(16) Merge<D> sh;
  const DecodeArgs& a = c.a;
  const int s = blockIdx.x % a.n_seqs, len = uniform(min(max(a.kv_len[s], 0), a.capacity));
  const Segment g = {(int)blockIdx.x / a.n_seqs, s, s, c.sh.group, 0, len, 0, len};
  Few<D, SRC, true> few(a, c.sh.group);
  few.start(g);
  // (so short a piece does not wait for a step of nothing: over codes 0.4 to 1 us of 7 to 20)
  if (few.steps(g) > 0) {
    int next[2];
    few.request_k(g, 0, few.pages, next);
    few.request_v(g, 0, next);
    few.there[0] = next[0];
    few.there[1] = next[1];
  }
  few.run(g, false, false, g, &sh, true, nullptr, nullptr);
}

// Few items (sequence, key / value head): each in parts of up to kMostUnits units of 128 tokens, the shortest that there are workgroups for.  A part is a
// workgroup's, whose wavefronts take every fourth step and add up in LDS: a quarter of the pieces for the join, and none that ends one sequence and
// begins another.  Lane i of a wavefront looks after sequences kEach i .. kEach i + kEach - 1.  False: parts would be longer, and nothing has been done.
template <int D, int SRC>
__device__ __forceinline__ bool few_items(const DecodeCall& c, Merge<D>& sh) {
  const DecodeArgs& a = c.a;
  constexpr int kUnit = kWaves * kStep, kEach = kFewSeqs / 64;
  const int lane = threadIdx.x & 63;
  int len[kEach], units[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int s = kEach * lane + i;
    len[i] = s < a.n_seqs ? min(max(a.kv_len[s], 0), a.capacity) : 0;
    sum += units[i] = (len[i] + kUnit - 1) / kUnit;
  }
  // units of a part; a call's units are below 2^29
  int share = max((wave_sum(sum) * a.n_kv_heads + kWorkgroups - 1) / kWorkgroups, 1), upto = 0;
  for (;; ++share) {
    if (share > kMostUnits) return false;
    sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += (units[i] + share - 1) / share;
    upto = wave_scan(sum);
    if (__builtin_amdgcn_readlane(upto, 63) * a.n_kv_heads <= kWorkgroups) break;
  }
  const int all = __builtin_amdgcn_readlane(upto, 63);      // parts of a head
  int first[kEach], parts[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    parts[i] = (units[i] + share - 1) / share;
    first[i] = i ? first[i ? i - 1 : 0] + parts[i ? i - 1 : 0] : upto - sum;
  }
  const Layout y = layout(a.n_seqs, a.n_kv_heads, c.sh.group, c.sh.n_passes, D);
  char* ws = static_cast<char*>(a.ws);
  // where the join finds every row's pieces
  if (threadIdx.x < 64)
    for (int h = blockIdx.x; h < a.n_kv_heads; h += gridDim.x)
#pragma unroll
      for (int i = 0; i < kEach; ++i)
        if (kEach * lane + i < a.n_seqs)
          reinterpret_cast<Meta*>(ws + y.meta)[h * a.n_seqs + kEach * lane + i] = make_int4(h * all + first[i], parts[i] == 1 ? -1 : parts[i], 0, 0);
  for (int number = blockIdx.x; number < all * a.n_kv_heads; number += gridDim.x) {
    const int h = number / all, at = number % all;
    int seq = 0, part = 0, n = 0, tokens = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      if (first[i] <= at && at < first[i] + parts[i]) {
        seq = kEach * lane + i;
        part = at - first[i];
        n = parts[i];
        tokens = len[i];
      }
    const int who = __builtin_ctzll(__ballot(n > 0));
    seq = __builtin_amdgcn_readlane(seq, who);
    part = __builtin_amdgcn_readlane(part, who);
    n = __builtin_amdgcn_readlane(n, who);
    tokens = __builtin_amdgcn_readlane(tokens, who);
    const Segment g = {h, seq, seq, c.sh.group, 0, tokens, part * share * kUnit, min((part + 1) * share * kUnit, tokens)};
    if (number >= (int)gridDim.x) __syncthreads();           // the last part's sums have been read
    Few<D, SRC, true> few(a, c.sh.group);
    few.start(g);
    few.run(g, true, false, g, &sh, n == 1, reinterpret_cast<float*>(ws + y.own_o) + (size_t)number * c.sh.group * D,
            reinterpret_cast<float2*>(ws + y.own_ml) + (size_t)number * c.sh.group);
  }
  return true;
}

template <int D, int SRC, int MODE>
__global__ __launch_bounds__(kThreads, 2) void k_attn_decode(DecodeCall c) {
  constexpr bool MANY = MODE >= MANY_ROWS, STREAM = MODE == STREAMED;
  __shared__ __align__(16) Shared<D, MODE> sh;
  const DecodeArgs& a = c.a;
  if constexpr (MODE == FEW_ITEMS)
    if (few_items<D, SRC>(c, sh.merge)) return;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const bool wide = MANY && c.sh.group > kFewRows;  // sequences' own parts have too many rows for the small body, too
  const int n_groups = MANY ? a.n_groups : 0, n_items = n_groups + a.n_seqs, n_many = wide ? n_items : n_groups;
  auto length = [&](int s) { return min(max(a.kv_len[s], 0), a.capacity); };
  auto tiles_of = [](int from, int to) { return to > from ? (to - (from & -kTile) + kTile - 1) / kTile : 0; };
  auto steps_of = [](int from, int to) { return to > from ? (to - (from & -kStep) + kStep - 1) / kStep : 0; };
  typedef Cost<SRC> C;
  const uint32_t tile_cost = wide ? kWaves : C::kTile, begin_cost = wide ? 2 * kWaves : C::kBegin;   // (a workgroup's border at every tile); see costs_fit
  // of a group's pass, or (wide) of a sequence's own part
  auto streamed = [&](int it) { return STREAM && it < n_groups && (a.behind[it] - a.first[it]) * c.sh.group <= kFewRows; };
  auto tile_cost_of = [&](int it) { return streamed(it) ? C::kTileStreamed : tile_cost; };
  auto begin_cost_of = [&](int it) { return streamed(it) ? C::kBeginStreamed : begin_cost; };
  auto many_cost = [&](int it, int from, int to) { return to > from ? begin_cost_of(it) + tiles_of(from, to) * tile_cost_of(it) : 0u; };
  auto own_cost = [&](int from, int to) { return wide ? many_cost(n_groups, from, to) : to > from ? C::kOwn + steps_of(from, to) : 0u; };
  // the tokens that are read once, of those that an expert's sequences share
  auto read_once = [](int prefix) { return shared_tokens(SRC == KV_PAGED_BLOCKS, prefix); };

  // ---- cost of every item, groups first
  for (int s = threadIdx.x; s < a.n_seqs; s += kThreads) sh.cum[n_groups + s] = own_cost(0, length(s));
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
        if (length(s) >= prefix) sh.cum[n_groups + s] = own_cost(read_once(prefix), length(s));
    if (lane == 0) {
      sh.group_src[g] = active ? src : -1;
      sh.cum[g] = active ? many_cost(g, 0, read_once(prefix)) * ((behind - first + c.sh.per_pass - 1) / c.sh.per_pass) : 0;
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
  auto shared_by = [&](int s, int len) {            // the tokens of a sequence (the same in all lanes) that a pass reads for it
    if (!MANY) return 0;
    const uint64_t who = __ballot(my_first <= s && s < my_behind && len >= my_prefix);
    return who ? read_once(__builtin_amdgcn_readlane(my_prefix, __builtin_ctzll(who))) : 0;
  };
  // ---- exclusive sums, in place
  {
    const int per = (n_items + kThreads - 1) / kThreads, lo = min((int)threadIdx.x * per, n_items), hi = min(lo + per, n_items);
    uint32_t sum = 0;
    for (int i = lo; i < hi; ++i) sum += sh.cum[i];
    const uint32_t run = (uint32_t)wave_scan((int)sum);
    if (lane == 63) sh.part[wave] = run;
    __syncthreads();
    uint32_t at = run - sum;
    for (int w = 0; w < wave; ++w) at += sh.part[w];
    for (int i = lo; i < hi; ++i) {
      const uint32_t v = sh.cum[i];
      sh.cum[i] = at;
      at += v;
    }
    if (threadIdx.x == kThreads - 1) sh.cum[n_items] = sh.part[0] + sh.part[1] + sh.part[2] + sh.part[3];
    __syncthreads();
  }
  // The line: what the larger body does, all heads, then, from a workgroup's border on, the rest, all heads.  Wavefront w has costs
  // [w chunk, (w + 1) chunk); of the larger body's part the workgroup's wavefronts do theirs together.
  const uint32_t many_head = uniform(sh.cum[n_many]), all_head = uniform(sh.cum[n_items]), few_head = all_head - many_head;
  const uint32_t many_all = many_head * a.n_kv_heads, few_all = few_head * a.n_kv_heads;
  const uint32_t shares = kWaves * (many_all && few_all && gridDim.x > 1 ? gridDim.x - 1 : gridDim.x);
  // (at least a tile's cost each, so that none of the workgroups that a pass is cut over is without a tile)
  const uint32_t chunk = max((uint32_t)(((uint64_t)many_all + few_all + shares - 1) / shares), MANY ? (tile_cost + kWaves - 1) / kWaves : 1u);
  const uint32_t each = kWaves * chunk, few_from = (many_all + each - 1) / each * each, all = few_from + few_all;
  auto end_of = [&](uint32_t number, uint32_t each, uint32_t most) { return (uint32_t)min((uint64_t)number * each, (uint64_t)most); };

  const Layout y = layout(a.n_seqs, a.n_kv_heads, c.sh.group, c.sh.n_passes, D);
  char* ws = static_cast<char*>(a.ws);
  float* own_o = reinterpret_cast<float*>(ws + y.own_o);
  float2* own_ml = reinterpret_cast<float2*>(ws + y.own_ml);

  // ---- the larger body's part: a tile is the workgroup's whose costs it begins in
  if constexpr (MANY) {
    const uint32_t end = end_of(blockIdx.x + 1, each, many_all);
    for (uint32_t u = end_of(blockIdx.x, each, many_all); u < end;) {
      const int h = uniform(u / many_head);
      const uint32_t in_head = u - h * many_head;
      int lo = 0, hi = n_many - 1;                  // last item that begins at or before u (those of no cost come before it)
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (sh.cum[mid] <= in_head) lo = mid; else hi = mid - 1;
      }
      const int it = uniform(lo);
      const uint32_t per_tile = uniform(tile_cost_of(it)), begin = uniform(begin_cost_of(it));
      auto tiles_before = [&](uint32_t cost) { return cost > begin ? (cost - begin + per_tile - 1) / per_tile : 0u; };   // that begin there
      uint32_t first = h * many_head + uniform(sh.cum[it]), behind = h * many_head + uniform(sh.cum[it + 1]);
      Segment g;
      bool direct = false;
      float* o;
      float2* ml;
      g.kvh = h;
      if (it < n_groups) {
        const uint32_t per_pass = many_cost(it, 0, read_once(a.prefix[it]));
        const int pass = uniform((u - first) / per_pass);
        first += pass * per_pass;
        behind = first + per_pass;
        g.seq = uniform(sh.group_src[it]);
        g.seq0 = a.first[it] + pass * c.sh.per_pass;
        g.rows = uniform(min(c.sh.per_pass, a.behind[it] - g.seq0) * c.sh.group);
        g.from = 0;
        g.to = read_once(a.prefix[it]);
        const size_t slot = (size_t)blockIdx.x + h * c.sh.n_passes + c.pass_base[it] + pass;
        o = reinterpret_cast<float*>(ws + y.prefix_o) + slot * kRowsPass * D;
        ml = reinterpret_cast<float2*>(ws + y.prefix_ml) + slot * kRowsPass;
      } else {
        const int s = it - n_groups;
        g.seq = g.seq0 = s;
        g.rows = c.sh.group;
        g.to = uniform(length(s));
        g.from = shared_by(s, g.to);
        const size_t slot = (size_t)blockIdx.x + (size_t)h * a.n_seqs + s;
        o = own_o + slot * c.sh.group * D;
        ml = own_ml + slot * c.sh.group;
      }
      const uint32_t stop = min(end, behind);
      const int tile0 = uniform(tiles_before(u - first)), tile1 = uniform(tiles_before(stop - first));
      u = stop;
      if (tile0 == tile1) continue;
      if (it >= n_groups) direct = g.from == 0 && tile0 == 0 && tile1 == (int)tiles_before(behind - first);
      g.t0 = (g.from & -kTile) + tile0 * kTile;
      g.t1 = min((g.from & -kTile) + tile1 * kTile, g.to);
      if constexpr (STREAM)
        if (streamed(it)) {
          static_assert(sizeof(Merge<D>) <= sizeof(sh.tiles), "LDS of both bodies");
          __syncthreads();                          // the last piece's reads of LDS are over
          Few<D, SRC, true> few(a, c.sh.group);
          few.start(g);
          few.run(g, true, false, g, &reinterpret_cast<Merge<D>&>(sh.tiles), false, o, ml);
          continue;
        }
      run_many<D, SRC>(a, c.sh.group, g, sh.tiles, direct, o, ml);
    }
    asm volatile("" ::: "memory");
  }

  // ---- the wavefront's own part, piece by piece
  if (!wide) {
    const uint32_t number = blockIdx.x * kWaves + wave;
    uint32_t u = max(end_of(number, chunk, all), few_from) - few_from;
    const uint32_t end = max(end_of(number + 1, chunk, all), few_from) - few_from;
    struct Piece {
      Segment g;
      bool direct;
      float* o;
      float2* ml;
    };
    int h = 0, it = n_groups;
    uint32_t first = 0;                             // cost before the item
    if (u < end) {
      h = uniform(u / few_head);
      const uint32_t in_head = u - h * few_head + many_head;
      int lo = n_groups, hi = n_items - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (sh.cum[mid] <= in_head) lo = mid; else hi = mid - 1;
      }
      it = uniform(lo);
    }
    auto next = [&](Piece& p) {
      while (u < end) {
        const uint32_t before = uniform(sh.cum[it]), cost = uniform(sh.cum[it + 1]) - before;
        first = h * few_head + before - many_head;
        const uint32_t stop = min(end, first + cost);
        if (cost && stop > first + C::kOwn) {
          const int s = it - n_groups;
          Segment& g = p.g;
          g.kvh = h;
          g.seq = g.seq0 = s;
          g.rows = c.sh.group;
          g.to = uniform(length(s));
          g.from = uniform(shared_by(s, g.to));
          const uint32_t from_step = u > first + C::kOwn ? u - first - C::kOwn : 0, to_step = stop - first - C::kOwn;
          p.direct = g.from == 0 && from_step == 0 && stop == first + cost;
          const size_t slot = (size_t)number + (size_t)h * a.n_seqs + s;
          p.o = own_o + slot * c.sh.group * D;
          p.ml = own_ml + slot * c.sh.group;
          g.t0 = uniform((g.from & -kStep) + from_step * kStep);
          g.t1 = uniform(min((int)((g.from & -kStep) + to_step * kStep), g.to));
        }
        const bool found = cost && stop > first + C::kOwn;
        u = stop;
        if (u == first + cost && ++it == n_items) {
          it = n_groups;
          ++h;
        }
        if (found) return true;
      }
      return false;
    };
    Piece p, then;
    Few<D, SRC, false> few(a, c.sh.group);
    for (int round = 0;; ++round) {
      const bool more = next(then);                 // while the first tokens of piece p are on their way
      if (round) few.run(p.g, round == 1, more, then.g, nullptr, p.direct, p.o, p.ml);
      else if (more) few.start(then.g);
      if (!more) break;
      p = then;
    }
  }

  // ---- where the join finds every row's pieces
  Meta* meta = reinterpret_cast<Meta*>(ws + y.meta);
  for (int i = blockIdx.x * kThreads + threadIdx.x; i < a.n_kv_heads * a.n_seqs; i += gridDim.x * kThreads) {
    const int h = i / a.n_seqs, s = i % a.n_seqs, it = n_groups + s;
    Meta w = make_int4(0, 0, 0, 0);
    for (int g = 0; g < n_groups; ++g) {
      if (s < a.first[g] || s >= a.behind[g]) continue;
      if (sh.group_src[g] >= 0 && length(s) >= a.prefix[g]) {
        const uint32_t n = many_cost(g, 0, read_once(a.prefix[g])), pass = (s - a.first[g]) / c.sh.per_pass;
        const uint32_t u0 = h * many_head + sh.cum[g] + pass * n, w0 = (u0 + begin_cost_of(g)) / each, w1 = (u0 + n - tile_cost_of(g)) / each;
        w.z = w0 + h * c.sh.n_passes + c.pass_base[g] + pass;
        w.w = (w1 - w0 + 1) | ((s - a.first[g]) % c.sh.per_pass * c.sh.group) << 16;
      }
      break;
    }
    const uint32_t cost = sh.cum[it + 1] - sh.cum[it];
    if (cost) {
      const uint32_t u0 = wide ? h * many_head + sh.cum[it] + begin_cost : few_from + h * few_head + sh.cum[it] - many_head + C::kOwn;
      const uint32_t last = u0 + cost - (wide ? begin_cost + tile_cost : C::kOwn + 1), by = wide ? each : chunk, w0 = u0 / by, w1 = last / by;
      w.x = w0 + i;
      w.y = w0 == w1 && w.w == 0 ? -1 : w1 - w0 + 1;
    }
    meta[i] = w;
  }
}

// One wavefront (W > 1: a workgroup of W, sharing out the pieces) per query row: the pieces of its prefix and its own, on one bound.
template <int D, int W>
__global__ __launch_bounds__(W == 1 ? kThreads : 64 * W) void k_join(DecodeCall c, bool scaled) {
  constexpr int E = D / 64;                          // dimensions per lane
  __shared__ float part[W][D];
  const DecodeArgs& a = c.a;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), group = c.sh.group;
  const int row = W > 1 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave;
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
    for (int k0 = W > 1 ? wave : 0; k0 < count; k0 += W * kBatch) {
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
  if constexpr (W > 1) {                             // all of them have the same bound and sum
#pragma unroll
    for (int e = 0; e < E; ++e) part[wave][E * lane + e] = x[e];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < W; ++w)
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] += part[w][E * lane + e];
  }
  const float inv = l == 0.0f ? 0.0f : (scaled ? a.v_scale[h] : 1.0f) / l;
  uint16_t* dst = a.out + (size_t)s * a.ld_out + (size_t)head * D + E * lane;
  if constexpr (E == 2) *reinterpret_cast<uint32_t*>(dst) = pack2(x[0] * inv, x[1] * inv);
  else *dst = (uint16_t)pack2(x[0] * inv, 0.0f);
}

// Whether passes of up to kFewRows rows stream their tokens, as sequences' own parts do, instead of bringing them to LDS for rows that are not there: where most
// tokens that a call shares are of such passes and, unless it is small, are more than a few tiles.  Prefixes of 2048 tokens, e4m3: 64 experts of two sequences, 40 heads of their
// own, 360 us (514 through LDS), 32 of 3, 32 heads over 8, 43 (50); bf16 with 16 heads of 64, 64 of two, 148 (172), but with 128
// dimensions as fast or slower (8 of 3, 40 heads: 82 and 75).
bool streaming_pays(const DecodeCall& c, int head_dim, int source) {
  if (c.sh.group > kFewRows || !(has_codes(source) || head_dim == 64)) return false;
  const bool small = c.a.n_seqs * c.a.n_kv_heads <= kFewItems;
  int64_t few = 0, more = 0;                        // tokens of such passes, of others
  for (int g = 0; g < c.a.n_groups; ++g) {
    const int n = c.a.behind[g] - c.a.first[g], prefix = c.a.prefix[g];
    if (n * c.sh.group <= kFewRows && (prefix >= kLeastStreamed || small)) few += prefix;
    else more += (int64_t)((n + c.sh.per_pass - 1) / c.sh.per_pass) * prefix;
  }
  return few > more;
}

template <int D, int SRC>
hipError_t launch(const DecodeCall& c, hipStream_t s) {
  const bool many = c.sh.group > kFewRows || c.a.n_groups > 0;
  if (!many && c.a.capacity <= kWholeTokens) {
    k_attn_decode_whole<D, SRC><<<(unsigned)(c.a.n_kv_heads * c.a.n_seqs), kThreads, 0, s>>>(c);
    return hipGetLastError();
  }
  // never more workgroups than steps there can be
  const int64_t most = (int64_t)c.a.n_kv_heads * (c.a.n_seqs + c.sh.n_passes) * ((c.a.capacity + kStep - 1) / kStep + 1);
  const unsigned grid = (unsigned)std::min<int64_t>(kWorkgroups, most);
  auto go = [&](auto mode) { k_attn_decode<D, SRC, decltype(mode)::value><<<grid, kThreads, 0, s>>>(c); };
  constexpr int kStreamed = has_codes(SRC) || D == 64 ? STREAMED : MANY_ROWS;
  if (many && streaming_pays(c, D, SRC)) go(std::integral_constant<int, kStreamed>{});
  else if (many) go(std::integral_constant<int, MANY_ROWS>{});
  else if (c.a.n_seqs * c.a.n_kv_heads <= kFewItems) go(std::integral_constant<int, FEW_ITEMS>{});
  else go(std::integral_constant<int, LINE>{});
  if (hipError_t e = hipGetLastError()) return e;
  const int rows = c.a.n_seqs * c.a.n_heads;
  if (rows <= 64) k_join<D, 16><<<rows, 1024, 0, s>>>(c, SRC == KV_PAGED_E4M3);
  else if (rows <= 1024) k_join<D, 4><<<rows, kThreads, 0, s>>>(c, SRC == KV_PAGED_E4M3);
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
