// C ABI of the serving operators: argument validation and launches.
// Declarations and contracts are in include/wavezip_serve.h.
#include <cmath>

#include "wz_serve.h"

using namespace wz;

namespace {

constexpr int kMostTokens = 1 << 24;
constexpr int64_t kMostGroups = 1 << 23;  // workgroups of a launch: their threads have to stay below 2^32

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
wz_status check_ptr(const void* p, uintptr_t align) {
  if (!p) return WZ_ERR_NULL;
  return aligned(p, align) ? WZ_OK : WZ_ERR_ALIGN;
}
wz_status from_hip(hipError_t e) { return e == hipSuccess ? WZ_OK : WZ_ERR_DEVICE; }

#define WZ_TRY(expr)                 \
  do {                               \
    const wz_status st_ = (expr);    \
    if (st_ != WZ_OK) return st_;    \
  } while (0)

wz_status check_cache_shape(const wz_cache* c) {
  if (!c) return WZ_ERR_NULL;
  const int P = c->page_size;
  if ((c->head_dim != 64 && c->head_dim != 128) || (P != 16 && P != 32 && P != 64 && P != 128) || c->kv_heads < 1 ||
      c->kv_heads > 256 || c->pages < 1)
    return WZ_ERR_SHAPE;
  return WZ_OK;
}
wz_status check_lengths(const wz_ragged* r) {
  if (!r) return WZ_ERR_NULL;
  if (r->batch < 1 || r->batch > 65536 || r->tokens < 0 || r->tokens >= kMostTokens || r->max_tokens < 0 ||
      r->max_tokens >= kMostTokens || r->max_kv < 0 || r->max_kv >= kMostTokens)
    return WZ_ERR_SHAPE;
  return WZ_OK;
}
wz_status check_batch_shape(const wz_ragged* r, const wz_cache& c) {
  WZ_TRY(check_lengths(r));
  return r->table_stride < 0 || int64_t(r->table_stride) * c.page_size < r->max_kv ? WZ_ERR_SHAPE : WZ_OK;
}
wz_status check_arrays(const wz_cache& c, const wz_ragged& r) {
  WZ_TRY(check_ptr(c.k, 16));
  WZ_TRY(check_ptr(c.v, 16));
  WZ_TRY(check_ptr(c.k_scale, 4));
  WZ_TRY(check_ptr(c.v_scale, 4));
  WZ_TRY(check_ptr(r.start, 4));
  WZ_TRY(check_ptr(r.kv_len, 4));
  return r.max_kv > 0 ? check_ptr(r.table, 4) : WZ_OK;
}
// Rows of `width` elements, `stride` apart; 8 elements are loaded at once.
wz_status check_rows(const void* p, int64_t stride, int64_t width) {
  WZ_TRY(check_ptr(p, 16));
  return stride < width || stride % 8 != 0 || stride > (int64_t(1) << 40) ? WZ_ERR_SHAPE : WZ_OK;
}
wz_status check_attention(const wz_cache* cache, const wz_ragged* batch, const wz_attention* cfg) {
  WZ_TRY(check_cache_shape(cache));
  WZ_TRY(check_batch_shape(batch, *cache));
  if (!cfg) return WZ_ERR_NULL;
  if (cfg->q_heads < 1 || cfg->q_heads % cache->kv_heads != 0 || cfg->q_heads / cache->kv_heads > 64)
    return WZ_ERR_SHAPE;
  if ((cfg->causal != 0 && cfg->causal != 1) || cfg->window < 0 || (cfg->window > 0 && !cfg->causal) ||
      !std::isfinite(cfg->scale))
    return WZ_ERR_PARAM;
  const AttendPlan p = attend_plan(*cache, *batch, cfg->q_heads, cfg->window);
  if (int64_t(p.slots) * cache->kv_heads > kMostGroups) return WZ_ERR_SHAPE;
  return WZ_OK;
}

wz_status check_states(const wz_states* s, const wz_ragged* r) {
  if (!s) return WZ_ERR_NULL;
  if ((s->head_dim != 64 && s->head_dim != 128) || s->heads < 1 || s->heads > 256 || s->slots < 1) return WZ_ERR_SHAPE;
  WZ_TRY(check_lengths(r));
  return int64_t(r->batch) * s->heads * (s->head_dim / 32) > kMostGroups ? WZ_ERR_SHAPE : WZ_OK;
}

// What the products of 8-bit integers have in common; `columns`: rows of all weights.
wz_status check_product(const int8_t* a, int64_t a_stride, const float* a_scale, int32_t M, int32_t N, int32_t K,
                        int64_t columns, const void* out, int64_t out_stride, int32_t out_dtype) {
  if (out_dtype != WZ_F32 && out_dtype != WZ_BF16) return WZ_ERR_DTYPE;
  if (M < 0 || M >= kMostTokens || N < 1 || columns >= kMostTokens || K < 16 || K > 65536 || K % 16 != 0 ||
      M * columns > int64_t(1) << 38)
    return WZ_ERR_SHAPE;
  if (M == 0) return WZ_OK;
  WZ_TRY(check_rows(a, a_stride, K));
  if (a_stride % 16 != 0 || a_stride > (1 << 22) || out_stride < N || out_stride > (int64_t(1) << 40))
    return WZ_ERR_SHAPE;
  WZ_TRY(check_ptr(a_scale, 4));
  return check_ptr(out, out_dtype == WZ_BF16 ? 2 : 4);
}
wz_status check_weights(const int8_t* w, int64_t w_stride, const float* w_scale, const float* bias, int32_t K) {
  WZ_TRY(check_rows(w, w_stride, K));
  if (w_stride % 16 != 0 || w_stride > (1 << 22)) return WZ_ERR_SHAPE;
  WZ_TRY(check_ptr(w_scale, 4));
  return bias && !aligned(bias, 4) ? WZ_ERR_ALIGN : WZ_OK;
}
bool is_activation(int32_t a) { return a >= WZ_ACT_NONE && a <= WZ_ACT_GELU_TANH; }

}  // namespace

extern "C" {

wz_status wz_cache_append(const wz_cache* cache, const wz_ragged* batch, const wz_rotation* rotation, const void* k,
                          int64_t k_stride, const void* v, int64_t v_stride, const void* q, int64_t q_stride,
                          int32_t q_heads, void* q_out, int64_t q_out_stride, int32_t in_dtype, void* stream) {
  WZ_TRY(check_cache_shape(cache));
  WZ_TRY(check_batch_shape(batch, *cache));
  if (in_dtype != WZ_F32 && in_dtype != WZ_BF16) return WZ_ERR_DTYPE;
  AppendArgs a{};
  a.cache = *cache, a.batch = *batch;
  if (rotation) {
    const wz_rotation& r = *rotation;
    if (r.rot_dim < 16 || r.rot_dim > cache->head_dim || r.rot_dim % 16 != 0 || r.max_pos < 1 || r.axes < 1 ||
        r.axes > 3)
      return WZ_ERR_SHAPE;
    if (r.interleaved != 0 && r.interleaved != 1) return WZ_ERR_PARAM;
    a.turn = r;
    if (r.axes < 3) a.turn.sections[2] = 0;
    if (r.axes > 1) {
      int64_t sum = 0;
      for (int i = 0; i < r.axes; ++i) {
        if (r.sections[i] < 0) return WZ_ERR_SHAPE;
        sum += r.sections[i];
      }
      if (sum != r.rot_dim / 2) return WZ_ERR_SHAPE;
    }
  }
  if (q && (q_heads < 1 || q_heads > 256 * 64)) return WZ_ERR_SHAPE;
  if (append_groups(*cache, *batch, q ? q_heads : 0) > kMostGroups) return WZ_ERR_SHAPE;
  // (without a new token to store there may still be queries to rotate)
  if (batch->tokens == 0 || (batch->max_tokens == 0 && !q)) return WZ_OK;
  WZ_TRY(check_arrays(*cache, *batch));
  if (rotation) {
    WZ_TRY(check_ptr(rotation->table, 16));
    WZ_TRY(check_ptr(rotation->positions, 4));
  }
  const int64_t width = int64_t(cache->kv_heads) * cache->head_dim;
  WZ_TRY(check_rows(k, k_stride, width));
  WZ_TRY(check_rows(v, v_stride, width));
  if (q) {
    WZ_TRY(check_rows(q, q_stride, int64_t(q_heads) * cache->head_dim));
    WZ_TRY(check_rows(q_out, q_out_stride, int64_t(q_heads) * cache->head_dim));
    if (q == q_out) return WZ_ERR_PARAM;
  }
  a.k = k, a.v = v, a.q = q, a.q_out = q_out;
  a.k_stride = k_stride, a.v_stride = v_stride, a.q_stride = q_stride, a.q_out_stride = q_out_stride;
  a.q_heads = q ? q_heads : 0;
  return from_hip(launch_append(a, in_dtype, static_cast<hipStream_t>(stream)));
}

size_t wz_attention_workspace_bytes(const wz_cache* cache, const wz_ragged* batch, const wz_attention* cfg) {
  if (check_attention(cache, batch, cfg) != WZ_OK) return 0;
  return attend_plan(*cache, *batch, cfg->q_heads, cfg->window).bytes;
}

wz_status wz_cache_attention(const wz_cache* cache, const wz_ragged* batch, const wz_attention* cfg, const void* q,
                             int64_t q_stride, void* out, int64_t out_stride, float* lse, void* ws, size_t ws_bytes,
                             void* stream) {
  WZ_TRY(check_attention(cache, batch, cfg));
  if (batch->tokens == 0 || batch->max_tokens == 0) return WZ_OK;
  WZ_TRY(check_arrays(*cache, *batch));
  const int64_t width = int64_t(cfg->q_heads) * cache->head_dim;
  WZ_TRY(check_rows(q, q_stride, width));
  WZ_TRY(check_rows(out, out_stride, width));
  if (lse && !aligned(lse, 4)) return WZ_ERR_ALIGN;
  const AttendPlan p = attend_plan(*cache, *batch, cfg->q_heads, cfg->window);
  AttendArgs a{};
  if (p.shared) {
    if (!ws) return WZ_ERR_NULL;
    if (!aligned(ws, 256) || ws_bytes < p.bytes) return WZ_ERR_WORKSPACE;
    a.part = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float*>(static_cast<char*>(ws) + p.part_bytes);
  }
  a.cache = *cache, a.batch = *batch, a.q = q, a.out = out, a.lse = lse;
  a.q_stride = q_stride, a.out_stride = out_stride;
  // (neither zero nor infinite: a masked score of -inf has to stay what it is)
  const float scale2 = cfg->scale * 1.44269504088896341f;
  a.scale2 = std::copysign(std::min(std::max(std::fabs(scale2), 0x1p-126f), 0x1.fffffep127f), scale2);
  // (no row sees kMostTokens places, so a longer window hides nothing either; places are above -kMostTokens, so a
  // place less this one stays in 32 bits)
  a.q_heads = cfg->q_heads, a.causal = cfg->causal, a.window = std::min(cfg->window, kMostTokens);
  a.blocks = p.blocks, a.workers = p.workers, a.shared = p.shared;
  a.block_rows = int(std::min(int64_t(p.block_rows), int64_t(batch->max_tokens) * (cfg->q_heads / cache->kv_heads)));
  return from_hip(launch_attend(a, p, static_cast<hipStream_t>(stream)));
}

wz_status wz_quantize_rows(const void* x, int64_t x_stride, int32_t rows, int32_t cols, int32_t in_dtype, int8_t* q,
                           int64_t q_stride, float* scale, void* stream) {
  if (in_dtype != WZ_F32 && in_dtype != WZ_BF16) return WZ_ERR_DTYPE;
  if (rows < 0 || rows >= kMostTokens || cols < 16 || cols > 65536 || cols % 16 != 0) return WZ_ERR_SHAPE;
  if (rows == 0) return WZ_OK;
  WZ_TRY(check_rows(x, x_stride, cols));
  WZ_TRY(check_rows(q, q_stride, cols));
  if (q_stride % 16 != 0) return WZ_ERR_SHAPE;
  WZ_TRY(check_ptr(scale, 4));
  return from_hip(launch_quantize(x, x_stride, rows, cols, in_dtype, q, q_stride, scale,
                                  static_cast<hipStream_t>(stream)));
}

wz_status wz_matmul_int(const int8_t* a, int64_t a_stride, const float* a_scale, const int8_t* w, int64_t w_stride,
                        const float* w_scale, const float* bias, int32_t M, int32_t N, int32_t K, void* out,
                        int64_t out_stride, int32_t out_dtype, void* stream) {
  if (out_dtype != WZ_F32 && out_dtype != WZ_BF16) return WZ_ERR_DTYPE;
  if (M < 0 || M >= kMostTokens || N < 1 || N >= kMostTokens || K < 16 || K > 65536 || K % 16 != 0 ||
      int64_t(M) * N > int64_t(1) << 38)
    return WZ_ERR_SHAPE;
  if (M == 0) return WZ_OK;
  WZ_TRY(check_rows(a, a_stride, K));
  WZ_TRY(check_rows(w, w_stride, K));
  if (a_stride % 16 != 0 || w_stride % 16 != 0 || a_stride > (1 << 22) || w_stride > (1 << 22) || out_stride < N ||
      out_stride > (int64_t(1) << 40))
    return WZ_ERR_SHAPE;
  WZ_TRY(check_ptr(a_scale, 4));
  WZ_TRY(check_ptr(w_scale, 4));
  WZ_TRY(check_ptr(out, out_dtype == WZ_BF16 ? 2 : 4));
  if (bias && !aligned(bias, 4)) return WZ_ERR_ALIGN;
  MatmulArgs p{a, w, a_scale, w_scale, bias, out, a_stride, w_stride, out_stride, M, N, K};
  return from_hip(launch_matmul(p, out_dtype, static_cast<hipStream_t>(stream)));
}

wz_status wz_matmul_int_epilogue(const int8_t* a, int64_t a_stride, const float* a_scale, const int8_t* w,
                                 int64_t w_stride, const float* w_scale, const float* bias, int32_t activation,
                                 const void* residual, int64_t residual_stride, int32_t M, int32_t N, int32_t K,
                                 void* out, int64_t out_stride, int32_t out_dtype, void* stream) {
  WZ_TRY(check_product(a, a_stride, a_scale, M, N, K, N, out, out_stride, out_dtype));
  if (!is_activation(activation)) return WZ_ERR_PARAM;
  if (M == 0) return WZ_OK;
  WZ_TRY(check_weights(w, w_stride, w_scale, bias, K));
  if (residual) {
    WZ_TRY(check_ptr(residual, out_dtype == WZ_BF16 ? 2 : 4));
    if (residual_stride < N || residual_stride > (int64_t(1) << 40)) return WZ_ERR_SHAPE;
    if (residual == out && residual_stride != out_stride) return WZ_ERR_PARAM;
  }
  MatmulArgs p{a, w, a_scale, w_scale, bias, out, a_stride, w_stride, out_stride, M, N, K};
  p.activation = activation, p.residual = residual, p.residual_stride = residual_stride;
  return from_hip(launch_matmul_epilogue(p, out_dtype, static_cast<hipStream_t>(stream)));
}

wz_status wz_gated_int(const int8_t* a, int64_t a_stride, const float* a_scale, const int8_t* gate,
                       int64_t gate_stride, const float* gate_scale, const float* gate_bias, const int8_t* up,
                       int64_t up_stride, const float* up_scale, const float* up_bias, int32_t activation, int32_t M,
                       int32_t N, int32_t K, void* out, int64_t out_stride, int32_t out_dtype, void* stream) {
  WZ_TRY(check_product(a, a_stride, a_scale, M, N, K, 2 * int64_t(N), out, out_stride, out_dtype));
  if (!is_activation(activation)) return WZ_ERR_PARAM;
  if (M == 0) return WZ_OK;
  WZ_TRY(check_weights(gate, gate_stride, gate_scale, gate_bias, K));
  WZ_TRY(check_weights(up, up_stride, up_scale, up_bias, K));
  MatmulArgs p{a, gate, a_scale, gate_scale, gate_bias, out, a_stride, gate_stride, out_stride, M, N, K};
  p.activation = activation, p.w2 = up, p.w2_stride = up_stride, p.w2_scale = up_scale, p.bias2 = up_bias;
  return from_hip(launch_gated(p, out_dtype, static_cast<hipStream_t>(stream)));
}

wz_status wz_norm_quantize(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride,
                           const float* weight, float eps, int32_t rows, int32_t cols, int32_t dtype, void* total,
                           int64_t total_stride, int8_t* q, int64_t q_stride, float* scale, void* stream) {
  if (dtype != WZ_F32 && dtype != WZ_BF16) return WZ_ERR_DTYPE;
  if (rows < 0 || rows >= kMostTokens || cols < 16 || cols > 65536 || cols % 16 != 0) return WZ_ERR_SHAPE;
  if (!(eps > 0) || !std::isfinite(eps)) return WZ_ERR_PARAM;
  if (rows == 0) return WZ_OK;
  WZ_TRY(check_rows(x, x_stride, cols));
  WZ_TRY(check_rows(q, q_stride, cols));
  if (q_stride % 16 != 0) return WZ_ERR_SHAPE;
  WZ_TRY(check_ptr(weight, 16));
  WZ_TRY(check_ptr(scale, 4));
  NormArgs p{x, residual, weight, nullptr, q, scale, x_stride, residual_stride, total_stride, q_stride, eps, rows, cols};
  if (residual) {
    WZ_TRY(check_rows(residual, residual_stride, cols));
    WZ_TRY(check_rows(total, total_stride, cols));
    if ((total == x && total_stride != x_stride) || (total == residual && total_stride != residual_stride))
      return WZ_ERR_PARAM;
    p.total = total;
  }
  return from_hip(launch_norm(p, dtype, static_cast<hipStream_t>(stream)));
}

size_t wz_decay_workspace_bytes(const wz_states* states, const wz_ragged* batch) {
  if (check_states(states, batch) != WZ_OK) return 0;
  return decay_plan(*states, *batch).bytes;
}

wz_status wz_decay_attention(const wz_states* states, const wz_ragged* batch, const int32_t* slot,
                             const float* log_decay, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, int32_t kv_heads, float scale, void* out,
                             int64_t out_stride, void* ws, size_t ws_bytes, void* stream) {
  WZ_TRY(check_states(states, batch));
  const int heads = states->heads, dim = states->head_dim;
  if (kv_heads < 1 || heads % kv_heads != 0) return WZ_ERR_SHAPE;
  if (!std::isfinite(scale)) return WZ_ERR_PARAM;
  if (batch->tokens == 0 || batch->max_tokens == 0) return WZ_OK;
  WZ_TRY(check_ptr(states->state, 16));
  WZ_TRY(check_ptr(batch->start, 4));
  WZ_TRY(check_ptr(batch->kv_len, 4));
  WZ_TRY(check_ptr(slot, 4));
  WZ_TRY(check_ptr(log_decay, 4));
  WZ_TRY(check_rows(q, q_stride, int64_t(heads) * dim));
  WZ_TRY(check_rows(k, k_stride, int64_t(kv_heads) * dim));
  WZ_TRY(check_rows(v, v_stride, int64_t(kv_heads) * dim));
  WZ_TRY(check_rows(out, out_stride, int64_t(heads) * dim));
  // (64 rows are addressed with 32 bits)
  if (std::max({q_stride, k_stride, v_stride}) > (1 << 22)) return WZ_ERR_SHAPE;
  if (out == q || out == k || out == v) return WZ_ERR_PARAM;
  DecayArgs p{*states, *batch, slot, log_decay, q, k, v, out, q_stride, k_stride, v_stride, out_stride, scale,
              heads / kv_heads};
  const DecayPlan plan = decay_plan(*states, *batch);
  p.runs = plan.runs, p.join = plan.join;
  if (plan.bytes) {
    if (!ws) return WZ_ERR_NULL;
    if (!aligned(ws, 256) || ws_bytes < plan.bytes) return WZ_ERR_WORKSPACE;
    p.part = static_cast<float*>(ws);
    p.goes_on = reinterpret_cast<int*>(static_cast<char*>(ws) + plan.state_bytes);
  }
  const auto s = static_cast<hipStream_t>(stream);
  return from_hip(plan.token ? launch_decay_token(p, s) : launch_decay_prompt(p, s));
}

}  // extern "C"
