// extern "C" entry points: argument validation on the host (before any HIP call), then launch.
#include "mes_attn.h"
#include "mes_bench.h"

#include <cstdarg>
#include <cstdio>
#include <vector>

namespace mes {

static thread_local char g_err[512] = "";
static thread_local hipEvent_t g_ev_start = nullptr, g_ev_stop = nullptr;

mes_status fail(mes_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return st;
}

mes_status check_hip(hipError_t e, const char* what) {
  if (e == hipSuccess) return MES_OK;
  return fail(MES_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
}

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static mes_status check_dims(int d_in, int d_out) {
  if (d_in <= 0 || d_out <= 0) return fail(MES_ERR_SHAPE, "d_in and d_out must be positive (got %d, %d)", d_in, d_out);
  if (d_in % 8 != 0) return fail(MES_ERR_SHAPE, "d_in must be a multiple of 8 (got %d)", d_in);
  if (d_out % 4 != 0) return fail(MES_ERR_SHAPE, "d_out must be a multiple of 4 (got %d)", d_out);
  return MES_OK;
}

static mes_status check_quant(int bits, int grid, int policy, bool allow_given) {
  if (bits < 1 || bits > 4) return fail(MES_ERR_BITS, "bits must be 1, 2, 3 or 4 (got %d)", bits);
  if (grid != MES_GRID_SYM && grid != MES_GRID_EQ1) return fail(MES_ERR_BITS, "unknown grid %d", grid);
  if (grid == MES_GRID_EQ1 && bits == 1) return fail(MES_ERR_BITS, "the Eq. 1 grid is undefined for bits = 1");
  if (policy < MES_STEP_GIVEN || policy > MES_STEP_MEANABS) return fail(MES_ERR_BITS, "unknown step policy %d", policy);
  if (policy == MES_STEP_GIVEN && !allow_given) return fail(MES_ERR_BITS, "step policy GIVEN is not valid here");
  if (policy == MES_STEP_MEANABS && bits != 1) return fail(MES_ERR_BITS, "step policy MEANABS needs bits = 1");
  return MES_OK;
}

}  // namespace mes

using namespace mes;

extern "C" {

const char* mes_last_error(void) { return g_err; }
int mes_layout_version(void) { return MES_LAYOUT_VERSION; }
int mes_long_segment_tokens(void) { return long_segment_tokens(); }

size_t mes_base_bytes(int d_in, int d_out) {
  if (d_in <= 0 || d_out <= 0) return 0;
  return (size_t)ceil_to(d_out, kRowPad) * ceil_to(d_in, kColPad) * 2;
}

size_t mes_codes_bytes(int d_in, int d_out, int bits) {
  if (d_in <= 0 || d_out <= 0 || bits < 1 || bits > 4) return 0;
  return (size_t)ceil_to(d_out, kRowPad) * ceil_to(d_in, kColPad) * bits / 8;
}

size_t mes_salient_bytes(int d_out, int k) {
  if (d_out <= 0 || k < 0) return 0;
  return (size_t)ceil_to(d_out, kRowPad) * ceil_to(k, kSalPad) * 2;
}

size_t mes_pack_workspace_bytes(void) { return 256; }

size_t mes_select_workspace_bytes(int n, int d_in, int d_out) {
  if (n <= 0 || d_in <= 0 || d_out <= 0) return 0;
  return (size_t)ceil_to(d_in, 32) * 8 + (size_t)ceil_to(d_out, 64) * 4 + (size_t)ceil_to(d_in, 32) * 4;
}

size_t mes_linear_multi_workspace_bytes(int d_in, const int32_t* d_out, int n_linears, int max_tokens) {
  if (d_in <= 0 || !d_out || n_linears < 1 || n_linears > MES_MAX_FUSED || max_tokens < 0) return 0;
  int d[MES_MAX_FUSED];
  for (int l = 0; l < n_linears; ++l) {
    if (d_out[l] <= 0) return 0;
    d[l] = d_out[l];
  }
  return linear_workspace_bytes(d_in, d, n_linears, max_tokens);
}

size_t mes_linear_workspace_bytes(int d_in, int d_out, int max_tokens) {
  const int32_t d = d_out;
  return mes_linear_multi_workspace_bytes(d_in, &d, 1, max_tokens);
}

mes_status mes_pack_base(const void* w, int d_in, int d_out, void* w_tiled_out, void* stream) {
  if (!w || !w_tiled_out) return fail(MES_ERR_NULL, "mes_pack_base: null pointer");
  if (mes_status st = check_dims(d_in, d_out)) return st;
  if (!aligned16(w) || !aligned16(w_tiled_out)) return fail(MES_ERR_ALIGN, "mes_pack_base: pointers must be 16-byte aligned");
  return check_hip(launch_pack_base((const uint16_t*)w, d_in, d_out, (uint16_t*)w_tiled_out, (hipStream_t)stream), "mes_pack_base");
}

mes_status mes_unpack_base(const void* w_tiled, int d_in, int d_out, void* w_out, void* stream) {
  if (!w_tiled || !w_out) return fail(MES_ERR_NULL, "mes_unpack_base: null pointer");
  if (mes_status st = check_dims(d_in, d_out)) return st;
  if (!aligned16(w_tiled) || !aligned16(w_out)) return fail(MES_ERR_ALIGN, "mes_unpack_base: pointers must be 16-byte aligned");
  return check_hip(launch_unpack_base((const uint16_t*)w_tiled, d_in, d_out, (uint16_t*)w_out, (hipStream_t)stream), "mes_unpack_base");
}

mes_status mes_select_salient(const float* delta, const float* x_calib, int n, int d_in, int d_out, int bits,
                              int grid, int step_policy, int k, int32_t* idx_out, double* score_out,
                              void* workspace, size_t workspace_bytes, void* stream) {
  if (!delta || !x_calib) return fail(MES_ERR_NULL, "mes_select_salient: null input");
  if (mes_status st = check_dims(d_in, d_out)) return st;
  if (n <= 0) return fail(MES_ERR_SHAPE, "mes_select_salient: n must be positive (got %d)", n);
  if (mes_status st = check_quant(bits, grid, step_policy, false)) return st;
  if (k < 0 || k > d_in) return fail(MES_ERR_SALIENT, "mes_select_salient: k = %d outside [0, %d]", k, d_in);
  if (k > 0 && !idx_out) return fail(MES_ERR_NULL, "mes_select_salient: idx_out is null");
  if (!workspace || workspace_bytes < mes_select_workspace_bytes(n, d_in, d_out))
    return fail(MES_ERR_WORKSPACE, "mes_select_salient: workspace needs %zu bytes", mes_select_workspace_bytes(n, d_in, d_out));
  if (!aligned16(workspace)) return fail(MES_ERR_ALIGN, "mes_select_salient: workspace must be 16-byte aligned");
  return check_hip(launch_select(delta, x_calib, n, d_in, d_out, bits, grid, step_policy, k, idx_out, score_out,
                                 workspace, (hipStream_t)stream), "mes_select_salient");
}

mes_status mes_pack_delta(const float* delta, int d_in, int d_out, const int32_t* salient_idx, int k, int bits,
                          int grid, int step_policy, const float* step_in, void* codes_out, float* step_out,
                          void* salient_out, void* workspace, size_t workspace_bytes, void* stream) {
  if (!delta || !codes_out || !step_out) return fail(MES_ERR_NULL, "mes_pack_delta: null pointer");
  if (mes_status st = check_dims(d_in, d_out)) return st;
  if (mes_status st = check_quant(bits, grid, step_policy, true)) return st;
  if (k < 0 || k > d_in) return fail(MES_ERR_SALIENT, "mes_pack_delta: k = %d outside [0, %d]", k, d_in);
  if (k > 0 && (!salient_idx || !salient_out)) return fail(MES_ERR_NULL, "mes_pack_delta: k > 0 needs salient_idx and salient_out");
  if (step_policy == MES_STEP_GIVEN && !step_in) return fail(MES_ERR_NULL, "mes_pack_delta: step policy GIVEN needs step_in");
  if (!aligned16(codes_out) || !aligned16(step_out) || (k > 0 && !aligned16(salient_out)))
    return fail(MES_ERR_ALIGN, "mes_pack_delta: outputs must be 16-byte aligned");
  if (!workspace || workspace_bytes < mes_pack_workspace_bytes())
    return fail(MES_ERR_WORKSPACE, "mes_pack_delta: workspace needs %zu bytes", mes_pack_workspace_bytes());
  hipStream_t s = (hipStream_t)stream;
  int* flag = reinterpret_cast<int*>(workspace);
  if (mes_status st = check_hip(launch_pack_delta(delta, d_in, d_out, salient_idx, k, bits, grid, step_policy, step_in,
                                                  (uint32_t*)codes_out, step_out, (uint16_t*)salient_out, flag, s),
                                "mes_pack_delta"))
    return st;
  int host_flag = 0;
  if (mes_status st = check_hip(hipMemcpyAsync(&host_flag, flag, sizeof(int), hipMemcpyDeviceToHost, s), "mes_pack_delta: flag copy"))
    return st;
  if (mes_status st = check_hip(hipStreamSynchronize(s), "mes_pack_delta: synchronize")) return st;
  if (host_flag) return fail(MES_ERR_SALIENT, "mes_pack_delta: salient_idx must be strictly ascending and inside [0, d_in)");
  return MES_OK;
}

static mes_status check_delta(const mes_delta* d, const char* who) {
  if (!d) return fail(MES_ERR_NULL, "%s: null descriptor", who);
  if (mes_status st = check_dims(d->d_in, d->d_out)) return st;
  if (mes_status st = check_quant(d->bits, d->grid, MES_STEP_GIVEN, true)) return st;
  if (d->layout_version != MES_LAYOUT_VERSION) return fail(MES_ERR_SHAPE, "%s: layout_version %d, library has %d", who, d->layout_version, MES_LAYOUT_VERSION);
  if (d->k < 0 || d->k > d->d_in) return fail(MES_ERR_SALIENT, "%s: k = %d outside [0, %d]", who, d->k, d->d_in);
  if (!d->codes || !d->step) return fail(MES_ERR_NULL, "%s: codes / step pointer is null", who);
  if (d->k > 0 && (!d->salient || !d->salient_idx)) return fail(MES_ERR_NULL, "%s: k > 0 needs salient and salient_idx", who);
  if (!aligned16(d->codes) || !aligned16(d->step) || (d->k > 0 && !aligned16(d->salient)))
    return fail(MES_ERR_ALIGN, "%s: codes, step and salient must be 16-byte aligned", who);
  return MES_OK;
}

mes_status mes_unpack_delta(const mes_delta* d, float* delta_hat_out, uint8_t* codes_out, void* stream) {
  if (mes_status st = check_delta(d, "mes_unpack_delta")) return st;
  if (!delta_hat_out && !codes_out) return fail(MES_ERR_NULL, "mes_unpack_delta: both outputs are null");
  return check_hip(launch_unpack_delta(*d, delta_hat_out, codes_out, (hipStream_t)stream), "mes_unpack_delta");
}

// mes_delta_linear_multi and, with gated != 0 (two layers: gate, up; one output at linears[0].y), mes_delta_linear_gated.
static mes_status run_linears(const char* who, const mes_linear* linears, int n_linears, int n_experts, const void* x, int T,
                              const int32_t* seg_offsets, void* workspace, size_t workspace_bytes, void* stream, int gated) {
  // the measurement hook is one-shot: this call consumes the events whichever way it returns
  const hipEvent_t ev_start = g_ev_start, ev_stop = g_ev_stop;
  g_ev_start = g_ev_stop = nullptr;
  if (n_linears < 1 || n_linears > MES_MAX_FUSED)
    return fail(MES_ERR_SHAPE, "%s: n_linears = %d outside [1, %d]", who, n_linears, MES_MAX_FUSED);
  if (n_experts < 1 || n_experts > MES_MAX_EXPERTS)
    return fail(MES_ERR_SHAPE, "%s: n_experts = %d outside [1, %d]", who, n_experts, MES_MAX_EXPERTS);
  if (T < 0) return fail(MES_ERR_SHAPE, "%s: T = %d is negative", who, T);
  if (!linears || !seg_offsets) return fail(MES_ERR_NULL, "%s: linears / seg_offsets is null", who);
  int32_t d_outs[MES_MAX_FUSED];
  for (int l = 0; l < n_linears; ++l) {
    if (!linears[l].experts) return fail(MES_ERR_NULL, "%s: experts is null", who);
    for (int e = 0; e < n_experts; ++e) {
      if (mes_status st = check_delta(&linears[l].experts[e], who)) return st;
      const mes_delta &a = linears[0].experts[0], &b = linears[l].experts[e];
      if (a.d_in != b.d_in || a.k != b.k || a.bits != b.bits || a.grid != b.grid || b.d_out != linears[l].experts[0].d_out)
        return fail(MES_ERR_SHAPE, "%s: expert %d of layer %d differs in d_in/d_out/k/bits/grid", who, e, l);
    }
    d_outs[l] = linears[l].experts[0].d_out;
  }
  if (seg_offsets[0] != 0) return fail(MES_ERR_SEGMENTS, "%s: seg_offsets[0] must be 0 (got %d)", who, seg_offsets[0]);
  for (int e = 0; e < n_experts; ++e)
    if (seg_offsets[e + 1] < seg_offsets[e]) return fail(MES_ERR_SEGMENTS, "%s: seg_offsets decreases at %d", who, e + 1);
  if (seg_offsets[n_experts] != T)
    return fail(MES_ERR_SEGMENTS, "%s: seg_offsets[%d] = %d, expected T = %d", who, n_experts, seg_offsets[n_experts], T);
  if (T == 0) return MES_OK;
  if (!x) return fail(MES_ERR_NULL, "%s: w_base / x / y is null", who);
  for (int l = 0; l < n_linears; ++l) {
    const bool has_y = !(gated && l > 0);   // the gated pair has one output
    if (!linears[l].w_base_tiled || (has_y && !linears[l].y)) return fail(MES_ERR_NULL, "%s: w_base / x / y is null", who);
    if (!aligned16(linears[l].w_base_tiled) || (has_y && !aligned16(linears[l].y)))
      return fail(MES_ERR_ALIGN, "%s: w_base, x and y must be 16-byte aligned", who);
  }
  if (!aligned16(x)) return fail(MES_ERR_ALIGN, "%s: w_base, x and y must be 16-byte aligned", who);
  if (gated && d_outs[0] != d_outs[1]) return fail(MES_ERR_SHAPE, "%s: gate and up projection differ in d_out (%d, %d)", who, d_outs[0], d_outs[1]);
  // the streaming path's share is what a call needs; the one-product scratch (sizes asked for with max_tokens >= 192)
  // is used when it is there
  const size_t need = gated ? gated_workspace_bytes(linears[0].experts[0].d_in, d_outs[0], 1)
                            : mes_linear_multi_workspace_bytes(linears[0].experts[0].d_in, d_outs, n_linears, 1);
  if (!workspace || workspace_bytes < need) return fail(MES_ERR_WORKSPACE, "%s: workspace needs %zu bytes", who, need);
  if (!aligned16(workspace)) return fail(MES_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  LinearCall c{linears, n_linears, n_experts, x, T, seg_offsets, workspace, workspace_bytes, ev_start, ev_stop, gated};
  return check_hip(launch_delta_linear(c, (hipStream_t)stream), who);
}

mes_status mes_delta_linear_multi(const mes_linear* linears, int n_linears, int n_experts, const void* x, int T,
                                  const int32_t* seg_offsets, void* workspace, size_t workspace_bytes, void* stream) {
  return run_linears("mes_delta_linear", linears, n_linears, n_experts, x, T, seg_offsets, workspace, workspace_bytes, stream, 0);
}

size_t mes_gated_workspace_bytes(int d_in, int d_out, int max_tokens) {
  if (d_in <= 0 || d_out <= 0 || max_tokens < 0) return 0;
  return gated_workspace_bytes(d_in, d_out, max_tokens);
}

mes_status mes_delta_linear_gated(const void* w_gate_tiled, const mes_delta* gate_experts, const void* w_up_tiled,
                                  const mes_delta* up_experts, int n_experts, const void* x, int T,
                                  const int32_t* seg_offsets, void* h, void* workspace, size_t workspace_bytes, void* stream) {
  const mes_linear pair[2] = {{w_gate_tiled, gate_experts, h}, {w_up_tiled, up_experts, nullptr}};
  return run_linears("mes_delta_linear_gated", pair, 2, n_experts, x, T, seg_offsets, workspace, workspace_bytes, stream, 1);
}

mes_status mes_delta_linear(const void* w_base_tiled, const mes_delta* experts, int n_experts, const void* x, int T,
                            const int32_t* seg_offsets, void* y, void* workspace, size_t workspace_bytes,
                            void* stream) {
  const mes_linear one{w_base_tiled, experts, y};
  return mes_delta_linear_multi(&one, 1, n_experts, x, T, seg_offsets, workspace, workspace_bytes, stream);
}

mes_status mes_time_next_call(void* start_event, void* stop_event) {
  if ((start_event == nullptr) != (stop_event == nullptr)) return fail(MES_ERR_NULL, "mes_time_next_call: give both events or neither");
  g_ev_start = (hipEvent_t)start_event;
  g_ev_stop = (hipEvent_t)stop_event;
  return MES_OK;
}

size_t mes_step_grad_workspace_bytes(int d_in, int d_out, int n_tokens) {
  if (d_in <= 0 || d_out <= 0 || n_tokens < 0) return 0;
  return step_grad_workspace_bytes(d_in, d_out, n_tokens);
}

mes_status mes_step_grad(const float* delta, int d_in, int d_out, const int32_t* salient_idx, int k, int bits, int grid,
                         const float* step, const void* x, int n_tokens, float* loss_out, float* grad_out,
                         void* workspace, size_t workspace_bytes, void* stream) {
  const hipEvent_t e0 = g_ev_start, e1 = g_ev_stop;   // one-shot measurement hook, consumed on every exit path
  g_ev_start = g_ev_stop = nullptr;
  if (!delta || !step || !loss_out || !grad_out) return fail(MES_ERR_NULL, "mes_step_grad: null pointer");
  if (mes_status st = check_dims(d_in, d_out)) return st;
  if (mes_status st = check_quant(bits, grid, MES_STEP_GIVEN, true)) return st;
  if (k < 0 || k > d_in) return fail(MES_ERR_SALIENT, "mes_step_grad: k = %d outside [0, %d]", k, d_in);
  if (k > 0 && !salient_idx) return fail(MES_ERR_NULL, "mes_step_grad: k > 0 needs salient_idx");
  if (n_tokens < 0) return fail(MES_ERR_SHAPE, "mes_step_grad: n_tokens must not be negative (got %d)", n_tokens);
  if (n_tokens > 0 && !x) return fail(MES_ERR_NULL, "mes_step_grad: x is null");
  if (!aligned16(delta) || !aligned16(step) || !aligned16(x))
    return fail(MES_ERR_ALIGN, "mes_step_grad: delta, step and x must be 16-byte aligned");
  if (!workspace || workspace_bytes < mes_step_grad_workspace_bytes(d_in, d_out, n_tokens))
    return fail(MES_ERR_WORKSPACE, "mes_step_grad: workspace needs %zu bytes", mes_step_grad_workspace_bytes(d_in, d_out, n_tokens));
  if (!aligned16(workspace)) return fail(MES_ERR_ALIGN, "mes_step_grad: workspace must be 16-byte aligned");
  return check_hip(launch_step_grad(delta, d_in, d_out, salient_idx, k, bits, grid, step, x, n_tokens, loss_out, grad_out,
                                    workspace, e0, e1, (hipStream_t)stream), "mes_step_grad");
}

mes_status mes_step_adamw(float* step, const float* grad, float* m, float* v, int n, int t, float lr, float beta1,
                          float beta2, float eps, float weight_decay, void* stream) {
  if (!step || !grad || !m || !v) return fail(MES_ERR_NULL, "mes_step_adamw: null pointer");
  if (n <= 0) return fail(MES_ERR_SHAPE, "mes_step_adamw: n must be positive (got %d)", n);
  if (t < 1) return fail(MES_ERR_SHAPE, "mes_step_adamw: t counts updates from 1 (got %d)", t);
  if (!(beta1 >= 0.0f && beta1 < 1.0f) || !(beta2 >= 0.0f && beta2 < 1.0f))
    return fail(MES_ERR_SHAPE, "mes_step_adamw: beta1 and beta2 must lie in [0, 1)");
  return check_hip(launch_adamw(step, grad, m, v, n, t, lr, beta1, beta2, eps, weight_decay, (hipStream_t)stream), "mes_step_adamw");
}

mes_status mes_copy_probe(void* dst, const void* src, size_t bytes, void* stream) {
  if (!dst || !src) return fail(MES_ERR_NULL, "mes_copy_probe: null buffer");
  if (bytes % 16 || ((uintptr_t)dst | (uintptr_t)src) % 16) return fail(MES_ERR_ALIGN, "mes_copy_probe: buffers and size must be multiples of 16 bytes");
  return check_hip(launch_copy_probe(dst, src, bytes, (hipStream_t)stream), "mes_copy_probe");
}

// ---- attention and its cache ---------------------------------------------------------------------------------

static mes_status check_heads(const char* who, int n_heads, int n_kv_heads, int head_dim) {
  if (head_dim != 64 && head_dim != 128) return fail(MES_ERR_SHAPE, "%s: head_dim must be 64 or 128 (got %d)", who, head_dim);
  if (n_kv_heads < 1 || n_heads < 1 || n_heads % n_kv_heads != 0 || n_heads / n_kv_heads > 64 || n_heads > 65535)
    return fail(MES_ERR_SHAPE, "%s: n_heads = %d must be 1 to 64 times n_kv_heads = %d", who, n_heads, n_kv_heads);
  return MES_OK;
}

// What indexes of 32 bits hold on the device: rows of a call (a launch has up to 2^32 threads), their distance, tokens of a page table
constexpr int kMaxRows = 0xffffff, kMaxStride = 1 << 26, kMaxTokens = 1 << 30;

static mes_status check_row_count(const char* who, int T) {
  if (T < 0 || T > kMaxRows) return fail(MES_ERR_SHAPE, "%s: T = %d outside [0, %d]", who, T, kMaxRows);
  return MES_OK;
}

static mes_status check_rows(const char* who, const char* what, const void* p, int ld, int heads, int head_dim) {
  if (!p) return fail(MES_ERR_NULL, "%s: %s is null", who, what);
  if (!aligned16(p)) return fail(MES_ERR_ALIGN, "%s: %s must be 16-byte aligned", who, what);
  if (ld < (int64_t)heads * head_dim || ld % 8 != 0 || ld > kMaxStride)
    return fail(MES_ERR_SHAPE, "%s: rows of %s are %d apart: a multiple of 8 in [%d, %d]", who, what, ld, heads * head_dim, kMaxStride);
  return MES_OK;
}

static mes_status check_kv(const char* who, const mes_kv* kv, int layer) {
  if (!kv) return fail(MES_ERR_NULL, "%s: kv is null", who);
  if (kv->dtype != MES_KV_BF16 && kv->dtype != MES_KV_E4M3 && kv->dtype != MES_KV_E4M3_BLOCKS) return fail(MES_ERR_BITS, "%s: unknown cache type %d", who, kv->dtype);
  if (kv->n_layers < 1 || kv->n_pages < 1) return fail(MES_ERR_SHAPE, "%s: n_layers = %d, n_pages = %d must be positive", who, kv->n_layers, kv->n_pages);
  if (kv->page_tokens < 16 || kv->page_tokens > 256 || (kv->page_tokens & (kv->page_tokens - 1)))
    return fail(MES_ERR_SHAPE, "%s: page_tokens must be 16, 32, 64, 128 or 256 (got %d)", who, kv->page_tokens);
  if (mes_status st = check_heads(who, kv->n_kv_heads, kv->n_kv_heads, kv->head_dim)) return st;
  if (!kv->k || !kv->v) return fail(MES_ERR_NULL, "%s: the cache's k / v is null", who);
  if (!aligned16(kv->k) || !aligned16(kv->v)) return fail(MES_ERR_ALIGN, "%s: the cache must be 16-byte aligned", who);
  if (kv->dtype == MES_KV_E4M3 && (!kv->k_scale || !kv->v_scale)) return fail(MES_ERR_NULL, "%s: an e4m3 cache needs k_scale and v_scale", who);
  if (kv->dtype == MES_KV_E4M3_BLOCKS && (!kv->k_exponent || !kv->v_exponent)) return fail(MES_ERR_NULL, "%s: a cache of blocks needs k_exponent and v_exponent", who);
  if (layer < 0 || layer >= kv->n_layers) return fail(MES_ERR_SHAPE, "%s: layer %d outside [0, %d)", who, layer, kv->n_layers);
  return MES_OK;
}

static mes_status check_seqs(const char* who, const mes_kv* kv, const mes_seqs* s, bool offsets) {
  if (!s) return fail(MES_ERR_NULL, "%s: seqs is null", who);
  if (s->n_seqs < 0 || s->n_seqs > MES_MAX_SEQS) return fail(MES_ERR_SHAPE, "%s: n_seqs = %d outside [0, %d]", who, s->n_seqs, MES_MAX_SEQS);
  if (s->n_seqs == 0) return MES_OK;
  if (!s->kv_len || !s->page_table || (offsets && !s->q_offsets)) return fail(MES_ERR_NULL, "%s: a pointer in seqs is null", who);
  if (s->table_pages < 1 || (int64_t)s->table_pages * kv->page_tokens > kMaxTokens)
    return fail(MES_ERR_SHAPE, "%s: table_pages = %d of %d tokens: 1 to %d tokens", who, s->table_pages, kv->page_tokens, kMaxTokens);
  return MES_OK;
}

static size_t kv_layer_bytes(const mes_kv& kv) {
  return (size_t)kv.n_pages * kv.n_kv_heads * kv.page_tokens * kv.head_dim * (kv.dtype == MES_KV_BF16 ? 2 : 1);
}
// first exponent of a layer, of k_exponent or v_exponent
static uint8_t* layer_exponents(const mes_kv& kv, uint8_t* of, int layer) {
  return of + (size_t)layer * kv.n_pages * kv.n_kv_heads * (kv.page_tokens / MES_KV_BLOCK);
}
static int source_of(const mes_kv& kv) { return kv.dtype == MES_KV_BF16 ? KV_PAGED : kv.dtype == MES_KV_E4M3 ? KV_PAGED_E4M3 : KV_PAGED_BLOCKS; }
static int log2_of(int v) { return 31 - __builtin_clz((unsigned)v); }

static mes_status check_angles(const char* who, const mes_angles& g, int head_dim) {
  if (!g.table) return fail(MES_ERR_NULL, "%s: the table of angles is null", who);
  if (!aligned16(g.table)) return fail(MES_ERR_ALIGN, "%s: the table of angles must be 16-byte aligned", who);
  if (g.dims < 16 || g.dims % 16 || g.dims > head_dim) return fail(MES_ERR_SHAPE, "%s: dims = %d: a multiple of 16 up to head_dim = %d", who, g.dims, head_dim);
  if (g.n_positions < 0) return fail(MES_ERR_SHAPE, "%s: n_positions = %d", who, g.n_positions);
  if (g.layout != MES_ROTARY_HALVES && g.layout != MES_ROTARY_PAIRS) return fail(MES_ERR_SHAPE, "%s: unknown layout %d", who, g.layout);
  return MES_OK;
}

static mes_status append(const char* who, bool fresh, const mes_kv* kv, int layer, const mes_seqs* seqs, const void* q, const void* k, const void* v, int T,
                         int n_heads, int ld_q, int ld_k, int ld_v, const mes_angles* angles, void* q_out, int ld_q_out, void* stream) {
  const float* rotary = angles ? angles->table : nullptr;
  if (mes_status st = check_kv(who, kv, layer)) return st;
  if (mes_status st = check_seqs(who, kv, seqs, false)) return st;
  if (mes_status st = check_row_count(who, T)) return st;
  if (!seqs->q_offsets && T > seqs->n_seqs) return fail(MES_ERR_SEGMENTS, "%s: %d rows of %d sequences without q_offsets", who, T, seqs->n_seqs);
  if (T == 0 || (seqs->n_seqs == 0 && !fresh)) return MES_OK;
  if (fresh && (!q || !q_out)) return fail(MES_ERR_NULL, "%s: q / q_out is null", who);
  if (fresh && q == q_out) return fail(MES_ERR_SHAPE, "%s: q_out is q", who);
  if ((q == nullptr) != (q_out == nullptr)) return fail(MES_ERR_NULL, "%s: give both of q and q_out or neither", who);
  if (q && !rotary) return fail(MES_ERR_NULL, "%s: q needs rotary", who);
  if (mes_status st = check_rows(who, "k", k, ld_k, kv->n_kv_heads, kv->head_dim)) return st;
  if (mes_status st = check_rows(who, "v", v, ld_v, kv->n_kv_heads, kv->head_dim)) return st;
  if (q) {
    if (n_heads < 1 || n_heads > 65535) return fail(MES_ERR_SHAPE, "%s: n_heads = %d", who, n_heads);
    if (mes_status st = check_rows(who, "q", q, ld_q, n_heads, kv->head_dim)) return st;
    if (mes_status st = check_rows(who, "q_out", q_out, ld_q_out, n_heads, kv->head_dim)) return st;
    if (q == q_out && ld_q != ld_q_out) return fail(MES_ERR_SHAPE, "%s: q_out is q with rows %d apart instead of %d", who, ld_q_out, ld_q);
  }
  const int capacity = seqs->n_seqs ? seqs->table_pages * kv->page_tokens : 0;   // no sequences: the table is not looked at
  if (angles) {
    if (mes_status st = check_angles(who, *angles, kv->head_dim)) return st;
    if (angles->n_positions < capacity)
      return fail(MES_ERR_SHAPE, "%s: rotary has %d positions, the page table has room for %d", who, angles->n_positions, capacity);
  }
  AppendArgs a{};
  a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v; a.q_out = (uint16_t*)q_out;
  a.rotary = rotary;
  if (angles) { a.dims = angles->dims; a.pairs = angles->layout == MES_ROTARY_PAIRS; }
  a.k_cache = kv->k; a.v_cache = kv->v;
  if (kv->dtype == MES_KV_E4M3) { a.k_scale = kv->k_scale; a.v_scale = kv->v_scale; }
  if (kv->dtype == MES_KV_E4M3_BLOCKS) { a.k_exponent = layer_exponents(*kv, kv->k_exponent, layer); a.v_exponent = layer_exponents(*kv, kv->v_exponent, layer); }
  a.q_offsets = seqs->q_offsets; a.kv_len = seqs->kv_len; a.page_table = seqs->page_table;
  a.T = T; a.layer = layer; a.n_pages = kv->n_pages; a.page_shift = log2_of(kv->page_tokens); a.n_heads = n_heads; a.n_kv_heads = kv->n_kv_heads;
  a.head_dim = kv->head_dim; a.n_seqs = seqs->n_seqs; a.table_pages = seqs->table_pages; a.capacity = capacity;
  a.ld_q = ld_q; a.ld_k = ld_k; a.ld_v = ld_v; a.ld_q_out = ld_q_out;
  a.fresh = fresh;
  return check_hip(launch_append(a, kv->dtype, (hipStream_t)stream), who);
}

mes_status mes_kv_append(const mes_kv* kv, int layer, const mes_seqs* seqs, const void* q, const void* k, const void* v, int T,
                         int n_heads, int ld_q, int ld_k, int ld_v, const float* rotary, int n_positions, void* q_out,
                         int ld_q_out, void* stream) {
  const mes_angles angles = {rotary, n_positions, kv ? kv->head_dim : 0, MES_ROTARY_HALVES};
  return append("mes_kv_append", false, kv, layer, seqs, q, k, v, T, n_heads, ld_q, ld_k, ld_v, rotary ? &angles : nullptr, q_out, ld_q_out, stream);
}

mes_status mes_kv_append_fresh(const mes_kv* kv, int layer, const mes_seqs* seqs, const void* q, const void* k, const void* v, int T,
                               int n_heads, int ld_q, int ld_k, int ld_v, const float* rotary, int n_positions, void* q_out,
                               int ld_q_out, void* stream) {
  const mes_angles angles = {rotary, n_positions, kv ? kv->head_dim : 0, MES_ROTARY_HALVES};
  return append("mes_kv_append_fresh", true, kv, layer, seqs, q, k, v, T, n_heads, ld_q, ld_k, ld_v, rotary ? &angles : nullptr, q_out, ld_q_out, stream);
}

mes_status mes_kv_append_angles(const mes_kv* kv, int layer, const mes_seqs* seqs, const void* q, const void* k, const void* v, int T,
                                int n_heads, int ld_q, int ld_k, int ld_v, const mes_angles* angles, void* q_out, int ld_q_out,
                                int fresh, void* stream) {
  if (fresh != 0 && fresh != 1) return fail(MES_ERR_SHAPE, "mes_kv_append_angles: fresh = %d", fresh);
  return append("mes_kv_append_angles", fresh == 1, kv, layer, seqs, q, k, v, T, n_heads, ld_q, ld_k, ld_v, angles, q_out, ld_q_out, stream);
}

mes_status mes_rotary_table(float* table, int n_positions, int dims, double base, int scaling, double factor, int context, double low,
                            double high, double magnitude, void* stream) {
  static const char who[] = "mes_rotary_table";
  if (n_positions < 0 || n_positions > 1 << 26) return fail(MES_ERR_SHAPE, "%s: n_positions = %d outside [0, %d]", who, n_positions, 1 << 26);
  if (dims < 16 || dims % 16 || dims > kMostTurned) return fail(MES_ERR_SHAPE, "%s: dims = %d: a multiple of 16 up to %d", who, dims, kMostTurned);
  if (scaling < MES_SCALING_NONE || scaling > MES_SCALING_BANDS) return fail(MES_ERR_SHAPE, "%s: unknown scaling %d", who, scaling);
  if (!(base > 0.0) || !std::isfinite(base)) return fail(MES_ERR_SHAPE, "%s: base must be positive and finite", who);
  if (!std::isfinite(magnitude)) return fail(MES_ERR_SHAPE, "%s: magnitude must be finite", who);
  if (scaling != MES_SCALING_NONE && (!(factor >= 1.0) || !std::isfinite(factor))) return fail(MES_ERR_SHAPE, "%s: factor must be at least 1 and finite", who);
  if (scaling == MES_SCALING_BANDS && (context < 1 || !(low >= 0.0) || !(high > low) || !std::isfinite(high)))
    return fail(MES_ERR_SHAPE, "%s: context must be positive and 0 <= low < high", who);
  if (n_positions == 0) return MES_OK;
  if (!table) return fail(MES_ERR_NULL, "%s: table is null", who);
  if (!aligned16(table)) return fail(MES_ERR_ALIGN, "%s: table must be 16-byte aligned", who);
  TableArgs a{};
  a.table = table;
  a.n_positions = n_positions;
  a.dims = dims;
  a.magnitude = magnitude;
  if (scaling == MES_SCALING_BASE) base *= std::pow(factor, dims / (dims - 2.0));
  for (int i = 0; i < dims / 2; ++i) {
    double f = std::pow(base, -2.0 * i / dims);
    if (scaling == MES_SCALING_LINEAR) f /= factor;
    if (scaling == MES_SCALING_BANDS) {
      const double keep = std::min(std::max((context * f / 6.283185307179586 - low) / (high - low), 0.0), 1.0);
      f *= keep + (1.0 - keep) / factor;
    }
    // a frequency that is not finite (a base near 0, to a power) has no angles
    if (!std::isfinite(f) || f > 1e6) return fail(MES_ERR_SHAPE, "%s: base %g gives dimension %d the frequency %g", who, base, i, f);
    a.frequency[i] = f;
  }
  return check_hip(launch_rotary_table(a, (hipStream_t)stream), who);
}

mes_status mes_rotary(const mes_angles* angles, const int32_t* positions, const void* q, const void* k, int T, int n_heads, int n_kv_heads,
                      int head_dim, int ld_q, int ld_k, int dtype, int transpose, void* q_out, int ld_q_out, void* k_out, int ld_k_out,
                      int fresh, void* stream) {
  static const char who[] = "mes_rotary";
  if (!angles) return fail(MES_ERR_NULL, "%s: angles is null", who);
  if (dtype != MES_ROWS_BF16 && dtype != MES_ROWS_FP32) return fail(MES_ERR_BITS, "%s: unknown type of rows %d", who, dtype);
  if (transpose != 0 && transpose != 1) return fail(MES_ERR_SHAPE, "%s: transpose = %d", who, transpose);
  if (fresh != 0 && fresh != 1) return fail(MES_ERR_SHAPE, "%s: fresh = %d", who, fresh);
  if (head_dim < 16 || head_dim % 16 || head_dim > kMostTurned) return fail(MES_ERR_SHAPE, "%s: head_dim = %d: a multiple of 16 up to %d", who, head_dim, kMostTurned);
  if (n_heads < 1 || n_heads > 65535 || (k && (n_kv_heads < 1 || n_kv_heads > 65535)))
    return fail(MES_ERR_SHAPE, "%s: n_heads = %d, n_kv_heads = %d: 1 to 65535", who, n_heads, n_kv_heads);
  if (mes_status st = check_angles(who, *angles, head_dim)) return st;
  if (mes_status st = check_row_count(who, T)) return st;
  if (T == 0) return MES_OK;
  if (!positions) return fail(MES_ERR_NULL, "%s: positions is null", who);
  if ((k == nullptr) != (k_out == nullptr)) return fail(MES_ERR_NULL, "%s: give both of k and k_out or neither", who);
  if (mes_status st = check_rows(who, "q", q, ld_q, n_heads, head_dim)) return st;
  if (mes_status st = check_rows(who, "q_out", q_out, ld_q_out, n_heads, head_dim)) return st;
  if (q == q_out && ld_q != ld_q_out) return fail(MES_ERR_SHAPE, "%s: q_out is q with rows %d apart instead of %d", who, ld_q_out, ld_q);
  if (k) {
    if (mes_status st = check_rows(who, "k", k, ld_k, n_kv_heads, head_dim)) return st;
    if (mes_status st = check_rows(who, "k_out", k_out, ld_k_out, n_kv_heads, head_dim)) return st;
    if (k == k_out && ld_k != ld_k_out) return fail(MES_ERR_SHAPE, "%s: k_out is k with rows %d apart instead of %d", who, ld_k_out, ld_k);
  }
  if (fresh && (q == q_out || (k && k == k_out))) return fail(MES_ERR_SHAPE, "%s: fresh outputs are not the inputs", who);
  RotaryArgs a{};
  a.q = q; a.k = k; a.q_out = q_out; a.k_out = k_out;
  a.positions = positions; a.table = angles->table;
  a.T = T; a.n_heads = n_heads; a.n_kv_heads = k ? n_kv_heads : 0; a.head_dim = head_dim;
  a.ld_q = ld_q; a.ld_k = ld_k; a.ld_q_out = ld_q_out; a.ld_k_out = ld_k_out;
  a.n_positions = angles->n_positions; a.dims = angles->dims; a.pairs = angles->layout == MES_ROTARY_PAIRS;
  a.sign = transpose ? -1.0f : 1.0f;
  a.fresh = fresh == 1;
  return check_hip(launch_rotary(a, dtype == MES_ROWS_FP32, (hipStream_t)stream), who);
}

mes_status mes_kv_read(const mes_kv* kv, int layer, const mes_seqs* seqs, int T, void* k, void* v, int ld_k, int ld_v, int fresh,
                       void* stream) {
  static const char who[] = "mes_kv_read";
  if (mes_status st = check_kv(who, kv, layer)) return st;
  if (mes_status st = check_seqs(who, kv, seqs, false)) return st;
  if (mes_status st = check_row_count(who, T)) return st;
  if (fresh != 0 && fresh != 1) return fail(MES_ERR_SHAPE, "%s: fresh = %d", who, fresh);
  if (!seqs->q_offsets && T > seqs->n_seqs) return fail(MES_ERR_SEGMENTS, "%s: %d rows of %d sequences without q_offsets", who, T, seqs->n_seqs);
  if (T == 0 || (seqs->n_seqs == 0 && !fresh)) return MES_OK;
  if (!k && !v) return fail(MES_ERR_NULL, "%s: k and v are null", who);
  if (k) if (mes_status st = check_rows(who, "k", k, ld_k, kv->n_kv_heads, kv->head_dim)) return st;
  if (v) if (mes_status st = check_rows(who, "v", v, ld_v, kv->n_kv_heads, kv->head_dim)) return st;
  if (k == v) return fail(MES_ERR_SHAPE, "%s: k is v", who);
  ReadArgs a{};
  a.k_cache = (const char*)kv->k + layer * kv_layer_bytes(*kv);
  a.v_cache = (const char*)kv->v + layer * kv_layer_bytes(*kv);
  if (kv->dtype == MES_KV_E4M3) { a.k_scale = kv->k_scale + (size_t)layer * kv->n_kv_heads; a.v_scale = kv->v_scale + (size_t)layer * kv->n_kv_heads; }
  if (kv->dtype == MES_KV_E4M3_BLOCKS) { a.k_exponent = layer_exponents(*kv, kv->k_exponent, layer); a.v_exponent = layer_exponents(*kv, kv->v_exponent, layer); }
  a.k = (uint16_t*)k; a.v = (uint16_t*)v;
  a.q_offsets = seqs->q_offsets; a.kv_len = seqs->kv_len; a.page_table = seqs->page_table;
  a.T = T; a.n_pages = kv->n_pages; a.page_shift = log2_of(kv->page_tokens); a.n_kv_heads = kv->n_kv_heads; a.head_dim = kv->head_dim;
  a.n_seqs = seqs->n_seqs; a.table_pages = seqs->table_pages; a.capacity = seqs->n_seqs ? seqs->table_pages * kv->page_tokens : 0;
  a.ld_k = ld_k; a.ld_v = ld_v;
  a.fresh = fresh == 1;
  return check_hip(launch_read(a, kv->dtype, (hipStream_t)stream), who);
}

size_t mes_attn_prompt_workspace_bytes(int T, int n_seqs, int n_heads, int n_kv_heads, int head_dim) {
  if (T < 0 || n_seqs < 0 || n_seqs > MES_MAX_SEQS || n_kv_heads < 1 || n_heads < 1 || n_heads % n_kv_heads || n_heads / n_kv_heads > 64 ||
      n_heads > 65535 || (head_dim != 64 && head_dim != 128))
    return 0;
  return attn_prompt_workspace_bytes(T, n_seqs, n_heads, n_kv_heads, head_dim);
}

static mes_status check_prompt_workspace(const char* who, int T, int n_seqs, int n_heads, int n_kv_heads, int head_dim, const void* workspace, size_t bytes) {
  if (!workspace) return MES_OK;
  const size_t need = attn_prompt_workspace_bytes(T, n_seqs, n_heads, n_kv_heads, head_dim);
  if (bytes < need) return fail(MES_ERR_WORKSPACE, "%s: workspace needs %zu bytes", who, need);
  if (!aligned16(workspace)) return fail(MES_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  return MES_OK;
}

mes_status mes_attn_prompt(const void* q, const void* k, const void* v, int T, int n_seqs, const int32_t* seq_offsets,
                           int n_heads, int n_kv_heads, int head_dim, int ld_q, int ld_k, int ld_v, float scale, void* out,
                           int ld_out, void* workspace, size_t workspace_bytes, void* stream) {
  static const char who[] = "mes_attn_prompt";
  if (mes_status st = check_heads(who, n_heads, n_kv_heads, head_dim)) return st;
  if (n_seqs < 0 || n_seqs > MES_MAX_SEQS) return fail(MES_ERR_SHAPE, "%s: n_seqs = %d outside [0, %d]", who, n_seqs, MES_MAX_SEQS);
  if (mes_status st = check_row_count(who, T)) return st;
  if (!(scale > 0.0f) || scale > 1e30f) return fail(MES_ERR_SHAPE, "%s: scale must be positive and finite", who);
  if (T == 0 || n_seqs == 0) return MES_OK;
  if (!seq_offsets) return fail(MES_ERR_NULL, "%s: seq_offsets is null", who);
  if (mes_status st = check_rows(who, "q", q, ld_q, n_heads, head_dim)) return st;
  if (mes_status st = check_rows(who, "k", k, ld_k, n_kv_heads, head_dim)) return st;
  if (mes_status st = check_rows(who, "v", v, ld_v, n_kv_heads, head_dim)) return st;
  if (mes_status st = check_rows(who, "out", out, ld_out, n_heads, head_dim)) return st;
  if (mes_status st = check_prompt_workspace(who, T, n_seqs, n_heads, n_kv_heads, head_dim, workspace, workspace_bytes)) return st;
  PromptArgs a{};
  a.ws = workspace;
  a.q = (const uint16_t*)q; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v; a.out = (uint16_t*)out;
  a.q_offsets = seq_offsets;
  a.T = T; a.n_seqs = n_seqs; a.n_heads = n_heads; a.n_kv_heads = n_kv_heads; a.head_dim = head_dim;
  a.ld_q = ld_q; a.ld_k = ld_k; a.ld_v = ld_v; a.ld_out = ld_out; a.scale = scale;
  return check_hip(launch_attn_prompt(a, KV_PACKED, (hipStream_t)stream), who);
}

mes_status mes_attn_extend(const mes_kv* kv, int layer, const mes_seqs* seqs, const void* q, int T, int n_heads, int ld_q,
                           float scale, void* out, int ld_out, void* workspace, size_t workspace_bytes, void* stream) {
  static const char who[] = "mes_attn_extend";
  if (mes_status st = check_kv(who, kv, layer)) return st;
  if (mes_status st = check_seqs(who, kv, seqs, true)) return st;
  if (mes_status st = check_heads(who, n_heads, kv->n_kv_heads, kv->head_dim)) return st;
  if (mes_status st = check_row_count(who, T)) return st;
  if (!(scale > 0.0f) || scale > 1e30f) return fail(MES_ERR_SHAPE, "%s: scale must be positive and finite", who);
  if (T == 0 || seqs->n_seqs == 0) return MES_OK;
  if (mes_status st = check_rows(who, "q", q, ld_q, n_heads, kv->head_dim)) return st;
  if (mes_status st = check_rows(who, "out", out, ld_out, n_heads, kv->head_dim)) return st;
  if (mes_status st = check_prompt_workspace(who, T, seqs->n_seqs, n_heads, kv->n_kv_heads, kv->head_dim, workspace, workspace_bytes)) return st;
  PromptArgs a{};
  a.ws = workspace;
  a.q = (const uint16_t*)q; a.out = (uint16_t*)out;
  a.k = (const uint16_t*)((const char*)kv->k + layer * kv_layer_bytes(*kv));
  a.v = (const uint16_t*)((const char*)kv->v + layer * kv_layer_bytes(*kv));
  if (kv->dtype == MES_KV_E4M3) { a.k_scale = kv->k_scale + (size_t)layer * kv->n_kv_heads; a.v_scale = kv->v_scale + (size_t)layer * kv->n_kv_heads; }
  if (kv->dtype == MES_KV_E4M3_BLOCKS) { a.k_exponent = layer_exponents(*kv, kv->k_exponent, layer); a.v_exponent = layer_exponents(*kv, kv->v_exponent, layer); }
  a.q_offsets = seqs->q_offsets; a.kv_len = seqs->kv_len; a.page_table = seqs->page_table;
  a.T = T; a.n_seqs = seqs->n_seqs; a.n_heads = n_heads; a.n_kv_heads = kv->n_kv_heads; a.head_dim = kv->head_dim;
  a.n_pages = kv->n_pages; a.page_shift = log2_of(kv->page_tokens); a.table_pages = seqs->table_pages;
  a.capacity = seqs->table_pages * kv->page_tokens;
  a.ld_q = ld_q; a.ld_out = ld_out; a.scale = scale;
  return check_hip(launch_attn_prompt(a, source_of(*kv), (hipStream_t)stream), who);
}

size_t mes_attn_decode_workspace_bytes(int n_seqs, int n_heads, int n_kv_heads, int head_dim) {
  if (n_seqs < 1 || n_seqs > MES_MAX_SEQS || n_kv_heads < 1 || n_heads < 1 || n_heads % n_kv_heads || n_heads / n_kv_heads > 64 ||
      n_heads > 65535 || (head_dim != 64 && head_dim != 128))
    return 0;
  return attn_decode_workspace_bytes(n_seqs, n_heads, n_kv_heads, head_dim);
}

mes_status mes_attn_decode(const mes_kv* kv, int layer, const mes_seqs* seqs, const void* q, int n_heads, int ld_q,
                           int n_experts, const int32_t* seg_offsets, const int32_t* prefix_len, float scale, void* out,
                           int ld_out, void* workspace, size_t workspace_bytes, void* stream) {
  static const char who[] = "mes_attn_decode";
  if (mes_status st = check_kv(who, kv, layer)) return st;
  if (mes_status st = check_seqs(who, kv, seqs, false)) return st;
  if (mes_status st = check_heads(who, n_heads, kv->n_kv_heads, kv->head_dim)) return st;
  if (!(scale > 0.0f) || scale > 1e30f) return fail(MES_ERR_SHAPE, "%s: scale must be positive and finite", who);
  if (seqs->n_seqs == 0) return MES_OK;
  if (mes_status st = check_rows(who, "q", q, ld_q, n_heads, kv->head_dim)) return st;
  if (mes_status st = check_rows(who, "out", out, ld_out, n_heads, kv->head_dim)) return st;
  if ((seg_offsets == nullptr) != (prefix_len == nullptr)) return fail(MES_ERR_NULL, "%s: give both of seg_offsets and prefix_len or neither", who);
  DecodeArgs a{};
  if (seg_offsets) {
    if (n_experts < 1 || n_experts > MES_MAX_EXPERTS) return fail(MES_ERR_SHAPE, "%s: n_experts = %d outside [1, %d]", who, n_experts, MES_MAX_EXPERTS);
    if (seg_offsets[0] != 0) return fail(MES_ERR_SEGMENTS, "%s: seg_offsets[0] must be 0 (got %d)", who, seg_offsets[0]);
    for (int e = 0; e < n_experts; ++e) {
      if (seg_offsets[e + 1] < seg_offsets[e]) return fail(MES_ERR_SEGMENTS, "%s: seg_offsets decreases at %d", who, e + 1);
      if (prefix_len[e] < 0) return fail(MES_ERR_SEGMENTS, "%s: prefix_len[%d] = %d is negative", who, e, prefix_len[e]);
    }
    if (seg_offsets[n_experts] != seqs->n_seqs)
      return fail(MES_ERR_SEGMENTS, "%s: seg_offsets[%d] = %d, expected n_seqs = %d", who, n_experts, seg_offsets[n_experts], seqs->n_seqs);
    // an expert with one sequence or without tokens that are read once shares nothing: only the others are handed on
    for (int e = 0; e < n_experts; ++e) {
      if (seg_offsets[e + 1] - seg_offsets[e] < 2 || shared_tokens(kv->dtype == MES_KV_E4M3_BLOCKS, prefix_len[e]) == 0) continue;
      a.first[a.n_groups] = seg_offsets[e];
      a.behind[a.n_groups] = seg_offsets[e + 1];
      a.prefix[a.n_groups++] = prefix_len[e];
    }
  }
  if ((int64_t)seqs->n_seqs * n_heads > kMaxRows)
    return fail(MES_ERR_SHAPE, "%s: %d sequences of %d heads are more than one call takes", who, seqs->n_seqs, n_heads);
  if (!decode_fits(seqs->n_seqs, kv->n_kv_heads, seqs->table_pages * kv->page_tokens))
    return fail(MES_ERR_SHAPE, "%s: %d page tables of %d pages are more than one call takes", who, seqs->n_seqs, seqs->table_pages);
  const size_t need = attn_decode_workspace_bytes(seqs->n_seqs, n_heads, kv->n_kv_heads, kv->head_dim);
  if (!workspace || workspace_bytes < need) return fail(MES_ERR_WORKSPACE, "%s: workspace needs %zu bytes", who, need);
  if (!aligned16(workspace)) return fail(MES_ERR_ALIGN, "%s: workspace must be 16-byte aligned", who);
  a.q = (const uint16_t*)q; a.out = (uint16_t*)out;
  a.k = (const char*)kv->k + layer * kv_layer_bytes(*kv);
  a.v = (const char*)kv->v + layer * kv_layer_bytes(*kv);
  if (kv->dtype == MES_KV_E4M3) { a.k_scale = kv->k_scale + (size_t)layer * kv->n_kv_heads; a.v_scale = kv->v_scale + (size_t)layer * kv->n_kv_heads; }
  if (kv->dtype == MES_KV_E4M3_BLOCKS) { a.k_exponent = layer_exponents(*kv, kv->k_exponent, layer); a.v_exponent = layer_exponents(*kv, kv->v_exponent, layer); }
  a.kv_len = seqs->kv_len; a.page_table = seqs->page_table; a.ws = workspace;
  a.n_seqs = seqs->n_seqs; a.n_heads = n_heads; a.n_kv_heads = kv->n_kv_heads; a.head_dim = kv->head_dim; a.n_pages = kv->n_pages;
  a.page_shift = log2_of(kv->page_tokens); a.table_pages = seqs->table_pages; a.capacity = seqs->table_pages * kv->page_tokens;
  a.ld_q = ld_q; a.ld_out = ld_out; a.scale = scale;
  return check_hip(launch_attn_decode(a, source_of(*kv), (hipStream_t)stream), who);
}

mes_status mes_kv_copy_pages(const mes_kv* kv, const int32_t* src, const int32_t* dst, int n, void* stream) {
  static const char who[] = "mes_kv_copy_pages";
  if (mes_status st = check_kv(who, kv, 0)) return st;
  if (n < 0 || n > kv->n_pages) return fail(MES_ERR_SHAPE, "%s: n = %d outside [0, %d]", who, n, kv->n_pages);
  if (n == 0) return MES_OK;
  if (!src || !dst) return fail(MES_ERR_NULL, "%s: src / dst is null", who);
  try {
    std::vector<int32_t> written(dst, dst + n);
    std::sort(written.begin(), written.end());
    for (int i = 0; i < n; ++i) {
      if (src[i] < 0 || src[i] >= kv->n_pages || dst[i] < 0 || dst[i] >= kv->n_pages)
        return fail(MES_ERR_PAGES, "%s: pair %d is page %d to page %d of %d", who, i, src[i], dst[i], kv->n_pages);
      if (i && written[i] == written[i - 1]) return fail(MES_ERR_PAGES, "%s: page %d is written twice", who, written[i]);
      if (std::binary_search(written.begin(), written.end(), src[i])) return fail(MES_ERR_PAGES, "%s: page %d is read and written", who, src[i]);
    }
  } catch (...) {
    return fail(MES_ERR_DEVICE, "%s: out of host memory", who);
  }
  return check_hip(launch_copy_pages(*kv, src, dst, n, (hipStream_t)stream), who);
}

}  // extern "C"
