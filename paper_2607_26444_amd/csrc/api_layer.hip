// C ABI of the layer around the exchange (declared in include/moe.h):
// argument validation and launches.  Nothing here allocates or synchronizes.

#include <limits.h>
#include <math.h>

#include "layer.h"

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

bool logit_dtype(int d) { return d == MOE_DTYPE_F32 || d == MOE_DTYPE_BF16; }

int route_shape(int64_t T, int k, int E, int dtype, int64_t pitch, int score, float scale) {
  if (T < 0 || k < 1 || k > MOE_MAX_K || E < 1 || E > MOE_MAX_EXPERTS || k > E) return MOE_EINVAL;
  if (T > 0 && T > (int64_t)INT32_MAX / k) return MOE_EINVAL;
  if (!logit_dtype(dtype) || (pitch != 0 && pitch < E) || pitch > INT32_MAX) return MOE_EINVAL;
  if (score != MOE_SCORE_SOFTMAX && score != MOE_SCORE_SIGMOID) return MOE_EINVAL;
  return isfinite(scale) ? MOE_OK : MOE_EINVAL;
}

// Sequences of the balance loss: whole ones.
int balance_sizes(int64_t T, int k, int E, int64_t seq_len) {
  if (T < 0 || T > (int64_t)INT32_MAX / k || E < 1 || E > MOE_MAX_EXPERTS || seq_len < 0 ||
      (seq_len > 0 && T % seq_len != 0))
    return MOE_EINVAL;
  return MOE_OK;
}

// Shape of 8-bit codes: their kind, and the scales of a row.  Of no rows codes and
// scales may be null: that is the address of an empty tensor.
int quant_shape(const void* q, const float* scales, int64_t rows, int dtype, int H, int& cols,
                moe::QuantKind& kind) {
  if ((rows > 0 && (!q || !scales)) ||
      (dtype != MOE_DTYPE_FP8_E4M3 && dtype != MOE_DTYPE_INT8) || cols < 0)
    return MOE_EINVAL;
  if (dtype == MOE_DTYPE_FP8_E4M3) {
    if (H % MOE_FP8_BLOCK != 0) return MOE_EALIGN;
    if (cols == 0) cols = H / MOE_FP8_BLOCK;
    if (cols != H / MOE_FP8_BLOCK) return MOE_EINVAL;
    kind = moe::kQuantFp8;
  } else {
    if (H % 16 != 0) return MOE_EALIGN;
    if (cols == 0) cols = 1;
    kind = moe::kQuantInt8;
  }
  return aligned(q, 16) && aligned(scales, 4) ? MOE_OK : MOE_EALIGN;
}

}  // namespace

extern "C" {

int moe_route(const void* logits, int dtype, int64_t logits_pitch, int64_t T, int k, int E,
              int score, const float* bias, int groups, int top_groups, int group_top, int renorm,
              float scale, const uint8_t* token_mask, int32_t* topk_idx, float* topk_w,
              void* stream) {
  const int rc = route_shape(T, k, E, dtype, logits_pitch, score, scale);
  if (rc) return rc;
  if (groups < 1 || groups > MOE_MAX_GROUPS || E % groups != 0 || top_groups < 1 ||
      top_groups > groups || group_top < 1 || group_top > 2 || k > top_groups * (E / groups))
    return MOE_EINVAL;
  if (T == 0) return MOE_OK;
  if (!logits || !topk_idx || !topk_w) return MOE_EINVAL;
  if (!aligned(logits, dtype == MOE_DTYPE_F32 ? 4 : 2) || !aligned(bias, 4) ||
      !aligned(topk_idx, 4) || !aligned(topk_w, 4))
    return MOE_EALIGN;
  moe::RouteArgs a;
  a.logits = logits;
  a.pitch = logits_pitch ? logits_pitch : E;
  a.tokens = T;
  a.f32 = dtype == MOE_DTYPE_F32;
  a.k = k;
  a.E = E;
  a.sigmoid = score == MOE_SCORE_SIGMOID;
  a.bias = bias;
  a.groups = groups;
  a.top_groups = top_groups;
  a.group_top = group_top;
  a.renorm = renorm != 0;
  a.scale = scale;
  a.token_mask = token_mask;
  a.topk_idx = topk_idx;
  a.topk_w = topk_w;
  return moe::hip_status(moe::launch_route(a, as_stream(stream)));
}

int moe_route_backward(const void* logits, int dtype, int64_t logits_pitch, int64_t T, int k,
                       int E, int score, int renorm, float scale, const int32_t* topk_idx,
                       const float* grad_w, void* grad_logits, void* stream) {
  const int rc = route_shape(T, k, E, dtype, logits_pitch, score, scale);
  if (rc) return rc;
  if (T == 0) return MOE_OK;
  if (!logits || !topk_idx || !grad_w || !grad_logits) return MOE_EINVAL;
  const uintptr_t size = dtype == MOE_DTYPE_F32 ? 4 : 2;
  if (!aligned(logits, size) || !aligned(grad_logits, size) || !aligned(topk_idx, 4) ||
      !aligned(grad_w, 4))
    return MOE_EALIGN;
  moe::RouteGradArgs a;
  a.logits = logits;
  a.pitch = logits_pitch ? logits_pitch : E;
  a.tokens = T;
  a.f32 = dtype == MOE_DTYPE_F32;
  a.k = k;
  a.E = E;
  a.sigmoid = score == MOE_SCORE_SIGMOID;
  a.renorm = renorm != 0;
  a.scale = scale;
  a.topk_idx = topk_idx;
  a.grad_w = grad_w;
  a.grad_logits = grad_logits;
  return moe::hip_status(moe::launch_route_backward(a, as_stream(stream)));
}

int moe_balance_workspace_bytes(int64_t T, int E, int64_t seq_len, size_t* out_bytes) {
  if (!out_bytes || balance_sizes(T, 1, E, seq_len)) return MOE_EINVAL;
  *out_bytes = moe::balance_shape(T, E, seq_len).bytes;
  return MOE_OK;
}

int moe_balance(const void* logits, int dtype, int64_t logits_pitch, int64_t T, int k, int E,
                int score, int64_t seq_len, const int32_t* topk_idx, const uint8_t* token_mask,
                int32_t* expert_count, int32_t* live_tokens, float* mean_score, float* loss,
                void* workspace, size_t workspace_bytes, void* stream) {
  int rc = route_shape(T, k, E, dtype, logits_pitch, score, 1.0f);
  if (!rc) rc = balance_sizes(T, k, E, seq_len);
  if (rc) return rc;
  const moe::BalanceShape s = moe::balance_shape(T, E, seq_len);
  if (s.seqs == 0) return MOE_OK;
  if ((T > 0 && (!logits || !topk_idx)) || !expert_count || !live_tokens) return MOE_EINVAL;
  if (!aligned(logits, dtype == MOE_DTYPE_F32 ? 4 : 2) || !aligned(topk_idx, 4) ||
      !aligned(expert_count, 4) || !aligned(live_tokens, 4) || !aligned(mean_score, 4) ||
      !aligned(loss, 4))
    return MOE_EALIGN;
  if (s.bytes > 0 && (!workspace || !aligned(workspace, 256) || workspace_bytes < s.bytes))
    return MOE_EWORKSPACE;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  moe::BalanceArgs a;
  a.logits = logits;
  a.pitch = logits_pitch ? logits_pitch : E;
  a.seq = s.seq;
  a.seqs = s.seqs;
  a.per = s.per;
  a.parts = s.parts;
  a.f32 = dtype == MOE_DTYPE_F32;
  a.k = k;
  a.E = E;
  a.sigmoid = score == MOE_SCORE_SIGMOID;
  a.topk_idx = topk_idx;
  a.token_mask = token_mask;
  a.expert_count = expert_count;
  a.live_tokens = live_tokens;
  a.mean_score = mean_score;
  a.loss = loss;
  a.partial = reinterpret_cast<float*>(ws);
  a.part_live = reinterpret_cast<int32_t*>(ws + s.live_at);
  a.tickets = reinterpret_cast<uint32_t*>(ws + s.ticket_at);
  a.pieces = reinterpret_cast<float*>(ws + s.piece_at);
  return moe::hip_status(moe::launch_balance(a, s, as_stream(stream)));
}

int moe_balance_backward(const void* logits, int dtype, int64_t logits_pitch, int64_t T, int E,
                         int score, int64_t seq_len, const uint8_t* token_mask,
                         const int32_t* expert_count, const int32_t* live_tokens,
                         const float* grad_loss, const void* grad_sum, void* grad_logits,
                         void* stream) {
  int rc = route_shape(T, 1, E, dtype, logits_pitch, score, 1.0f);
  if (!rc) rc = balance_sizes(T, 1, E, seq_len);
  if (rc) return rc;
  if (T == 0) return MOE_OK;
  if (!logits || !expert_count || !live_tokens || !grad_loss || !grad_logits) return MOE_EINVAL;
  const uintptr_t size = dtype == MOE_DTYPE_F32 ? 4 : 2;
  if (!aligned(logits, size) || !aligned(grad_sum, size) || !aligned(grad_logits, size) ||
      !aligned(expert_count, 4) || !aligned(live_tokens, 4) || !aligned(grad_loss, 4))
    return MOE_EALIGN;
  moe::BalanceGradArgs a;
  a.logits = logits;
  a.pitch = logits_pitch ? logits_pitch : E;
  a.seq = seq_len ? seq_len : T;
  a.seqs = T / a.seq;
  a.f32 = dtype == MOE_DTYPE_F32;
  a.E = E;
  moe::balance_grad_parts(a);
  a.sigmoid = score == MOE_SCORE_SIGMOID;
  a.token_mask = token_mask;
  a.expert_count = expert_count;
  a.live_tokens = live_tokens;
  a.grad_loss = grad_loss;
  a.grad_sum = grad_sum;
  a.grad_logits = grad_logits;
  return moe::hip_status(moe::launch_balance_backward(a, as_stream(stream)));
}

int moe_rmsnorm(const uint16_t* x, int64_t x_pitch, const void* residual, int residual_dtype,
                int64_t residual_pitch, const void* weight, int weight_dtype, float eps, int64_t T,
                int H, void* sum_out, uint16_t* y, int q_dtype, void* q, float* q_scales,
                int scale_cols, float* rstd, void* stream) {
  if (T < 0 || T > INT32_MAX || H < 1 || H > MOE_MAX_ROW || !(eps >= 0.0f)) return MOE_EINVAL;
  if (!logit_dtype(weight_dtype) || !weight || (residual && !logit_dtype(residual_dtype)) ||
      (T > 0 && sum_out && !residual))
    return MOE_EINVAL;
  if ((x_pitch != 0 && x_pitch < H) || (residual_pitch != 0 && residual_pitch < H) ||
      x_pitch > INT32_MAX || residual_pitch > INT32_MAX)
    return MOE_EINVAL;
  moe::NormArgs a = {};                          // no codes
  const int rc = q ? quant_shape(q, q_scales, T, q_dtype, H, scale_cols, a.quant) : MOE_OK;
  if (rc) return rc;
  const bool rf = residual && residual_dtype == MOE_DTYPE_F32;
  if (H % 8 != 0 || x_pitch % 8 != 0 || residual_pitch % (rf ? 4 : 8) != 0 || !aligned(x, 16) ||
      !aligned(residual, 16) || !aligned(weight, 16) || !aligned(sum_out, 16) || !aligned(y, 16) ||
      !aligned(rstd, 4))
    return MOE_EALIGN;
  if (sum_out && sum_out == residual && residual_pitch != 0 && residual_pitch != H)
    return MOE_EINVAL;
  if (T == 0) return MOE_OK;
  if (!x || (!sum_out && !y && !q && !rstd)) return MOE_EINVAL;
  a.x = reinterpret_cast<const uint8_t*>(x);
  a.x_pitch = 2 * (x_pitch ? x_pitch : H);
  a.residual = static_cast<const uint8_t*>(residual);
  a.residual_f32 = rf;
  a.residual_pitch = (rf ? 4 : 2) * (residual_pitch ? residual_pitch : H);
  a.weight = static_cast<const uint8_t*>(weight);
  a.weight_f32 = weight_dtype == MOE_DTYPE_F32;
  a.eps = eps;
  a.rows = T;
  a.H = H;
  a.sum_out = static_cast<uint8_t*>(sum_out);
  a.y = reinterpret_cast<uint8_t*>(y);
  a.stream_y = T * H >= (int64_t)32 << 20;
  a.q = static_cast<uint8_t*>(q);
  a.q_scales = q_scales;
  a.scale_cols = scale_cols;
  a.rstd = rstd;
  return moe::hip_status(moe::launch_norm(a, as_stream(stream)));
}

int moe_quantize(const uint16_t* x, int64_t x_pitch, int64_t rows, int H, const int32_t* row_src,
                 int q_dtype, void* q, float* q_scales, int scale_cols, void* stream) {
  if (rows < 0 || rows > INT32_MAX || H < 1 || H > MOE_MAX_ROW ||
      (x_pitch != 0 && x_pitch < H) || x_pitch > INT32_MAX)
    return MOE_EINVAL;
  moe::NormArgs a = {};
  const int rc = quant_shape(q, q_scales, rows, q_dtype, H, scale_cols, a.quant);
  if (rc) return rc;
  if (H % 8 != 0 || x_pitch % 8 != 0 || !aligned(x, 16) || !aligned(row_src, 4))
    return MOE_EALIGN;
  if (rows == 0) return MOE_OK;
  if (!x) return MOE_EINVAL;
  a.x = reinterpret_cast<const uint8_t*>(x);
  a.x_pitch = 2 * (x_pitch ? x_pitch : H);
  a.rows = rows;
  a.H = H;
  a.row_src = row_src;
  a.q = static_cast<uint8_t*>(q);
  a.q_scales = q_scales;
  a.scale_cols = scale_cols;
  return moe::hip_status(moe::launch_norm(a, as_stream(stream)));
}

int moe_rmsnorm_backward_workspace_bytes(int64_t T, int H, size_t* out_bytes) {
  if (!out_bytes || T < 0 || T > INT32_MAX || H < 1 || H > MOE_MAX_ROW) return MOE_EINVAL;
  if (H % 8 != 0) return MOE_EALIGN;
  *out_bytes = (size_t)moe::norm_grad_parts(T, H) * H * sizeof(float);
  return MOE_OK;
}

int moe_rmsnorm_backward(const uint16_t* grad_y, const void* h, int h_dtype, const float* rstd,
                         const void* weight, int weight_dtype, const void* grad_sum, int64_t T,
                         int H, void* grad_x, float* grad_weight, void* workspace,
                         size_t workspace_bytes, void* stream) {
  size_t need = 0;
  const int rc = moe_rmsnorm_backward_workspace_bytes(T, H, &need);
  if (rc) return rc;
  if (!logit_dtype(h_dtype) || !logit_dtype(weight_dtype) || !weight) return MOE_EINVAL;
  if (T > 0 && (!grad_y || !h || !rstd || !grad_x)) return MOE_EINVAL;
  if (!aligned(grad_y, 16) || !aligned(h, 16) || !aligned(rstd, 4) || !aligned(weight, 16) ||
      !aligned(grad_sum, 16) || !aligned(grad_x, 16) || !aligned(grad_weight, 4))
    return MOE_EALIGN;
  if (grad_weight && need > 0 &&
      (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
    return MOE_EWORKSPACE;
  moe::NormGradArgs a;
  a.grad_y = reinterpret_cast<const uint8_t*>(grad_y);
  a.h = static_cast<const uint8_t*>(h);
  a.h_f32 = h_dtype == MOE_DTYPE_F32;
  a.weight_f32 = weight_dtype == MOE_DTYPE_F32;
  a.rstd = rstd;
  a.weight = static_cast<const uint8_t*>(weight);
  a.grad_sum = static_cast<const uint8_t*>(grad_sum);
  a.rows = T;
  a.H = H;
  a.grad_x = static_cast<uint8_t*>(grad_x);
  a.grad_weight = grad_weight;
  a.partial = static_cast<float*>(workspace);
  if (T == 0 && !grad_weight) return MOE_OK;
  return moe::hip_status(moe::launch_norm_backward(a, as_stream(stream)));
}

int moe_expert_matmul(const int8_t* a, const float* a_scales, int a_scale_pitch, int64_t rows,
                      const int8_t* w, const float* w_scales, int E, int N, int K,
                      const int32_t* expert_offset, const int32_t* expert_count, int act,
                      uint16_t* y, void* stream) {
  if (rows < 0 || rows > INT32_MAX || E < 1 || E > MOE_MAX_EXPERTS || N < 1 || K < 1 ||
      K > MOE_MAX_DEPTH || a_scale_pitch < 0)
    return MOE_EINVAL;
  if (act != MOE_ACT_NONE && act != MOE_ACT_SWIGLU) return MOE_EINVAL;
  if ((!expert_offset && (E != 1 || expert_count)) || !w || !w_scales) return MOE_EINVAL;
  const bool swiglu = act == MOE_ACT_SWIGLU;
  if (K % 16 != 0 || N % (swiglu ? 16 : 8) != 0 || !aligned(a, 16) || !aligned(w, 16) ||
      !aligned(y, 16) || !aligned(a_scales, 4) || !aligned(w_scales, 4) ||
      !aligned(expert_offset, 4) || !aligned(expert_count, 4))
    return MOE_EALIGN;
  if (rows == 0) return MOE_OK;
  if (!a || !a_scales || !y) return MOE_EINVAL;
  moe::MatmulArgs m;
  m.a = reinterpret_cast<const uint8_t*>(a);
  m.a_scales = a_scales;
  m.a_scale_pitch = a_scale_pitch ? a_scale_pitch : 1;
  m.E = E;
  m.rows = rows;
  m.w = reinterpret_cast<const uint8_t*>(w);
  m.w_scales = w_scales;
  m.N = N;
  m.K = K;
  m.offset = expert_offset;
  m.count = expert_count;
  m.swiglu = swiglu;
  m.y = y;
  return moe::hip_status(moe::launch_matmul(m, as_stream(stream)));
}

int moe_quantize_mx(const uint16_t* x, int64_t x_pitch, int64_t rows, int H,
                    const int32_t* row_src, uint8_t* q, int64_t q_pitch, uint8_t* q_scales,
                    int64_t scale_pitch, uint16_t* values, void* stream) {
  if (rows < 0 || rows > INT32_MAX || H < 1 || H > MOE_MAX_DEPTH || (x_pitch != 0 && x_pitch < H) ||
      x_pitch > INT32_MAX)
    return MOE_EINVAL;
  if (H % MOE_MX_BLOCK != 0) return MOE_EALIGN;
  const int64_t packed = moe::mx_scale_bytes(H);
  if ((q_pitch != 0 && q_pitch < H / 2) || q_pitch > INT32_MAX ||
      (scale_pitch != 0 && scale_pitch < packed) || scale_pitch > INT32_MAX)
    return MOE_EINVAL;
  if (x_pitch % 8 != 0 || q_pitch % 16 != 0 || scale_pitch % 4 != 0 || !aligned(x, 16) ||
      !aligned(row_src, 4) || !aligned(q, 16) || !aligned(q_scales, 4) || !aligned(values, 16))
    return MOE_EALIGN;
  if (rows == 0) return MOE_OK;
  if (!x || !q || !q_scales) return MOE_EINVAL;
  moe::MxQuantArgs a;
  a.x = reinterpret_cast<const uint8_t*>(x);
  a.x_pitch = 2 * (x_pitch ? x_pitch : H);
  a.rows = rows;
  a.H = H;
  a.row_src = row_src;
  a.q = q;
  a.q_pitch = q_pitch ? q_pitch : H / 2;
  a.scales = q_scales;
  a.scale_pitch = scale_pitch ? scale_pitch : packed;
  a.values = reinterpret_cast<uint8_t*>(values);
  return moe::hip_status(moe::launch_quantize_mx(a, as_stream(stream)));
}

int moe_expert_matmul_mx(const uint8_t* a, int a_pitch, const uint8_t* a_scales, int a_scale_pitch,
                         int64_t rows, const uint8_t* w, const uint8_t* w_scales, int E, int N,
                         int K, const int32_t* expert_offset, const int32_t* expert_count, int act,
                         uint16_t* y, void* stream) {
  if (rows < 0 || rows > INT32_MAX || E < 1 || E > MOE_MAX_EXPERTS || N < 1 ||
      N > MOE_MAX_MX_CHANNELS || K < 1 || K > MOE_MAX_DEPTH)
    return MOE_EINVAL;
  if (act != MOE_ACT_NONE && act != MOE_ACT_SWIGLU) return MOE_EINVAL;
  if ((!expert_offset && (E != 1 || expert_count)) || !w || !w_scales) return MOE_EINVAL;
  const bool swiglu = act == MOE_ACT_SWIGLU;
  if (K % MOE_MX_BLOCK != 0) return MOE_EALIGN;
  const int packed = moe::mx_scale_bytes(K);
  if ((a_pitch != 0 && a_pitch < K / 2) || a_pitch > MOE_MAX_MX_PITCH ||
      (a_scale_pitch != 0 && a_scale_pitch < packed) || a_scale_pitch > MOE_MAX_MX_PITCH)
    return MOE_EINVAL;
  if (N % (swiglu ? 16 : 8) != 0 || a_pitch % 16 != 0 || a_scale_pitch % 4 != 0 || !aligned(a, 16) ||
      !aligned(w, 16) || !aligned(y, 16) || !aligned(a_scales, 4) || !aligned(w_scales, 4) ||
      !aligned(expert_offset, 4) || !aligned(expert_count, 4))
    return MOE_EALIGN;
  if (rows == 0) return MOE_OK;
  if (!a || !a_scales || !y) return MOE_EINVAL;
  moe::MatmulMxArgs m;
  m.rows = rows;
  m.E = E;
  m.N = N;
  m.K = K / 2;
  m.swiglu = swiglu;
  m.offset = expert_offset;
  m.count = expert_count;
  m.a = a;
  m.a_scales = a_scales;
  m.a_pitch = a_pitch ? a_pitch : K / 2;
  m.a_scale_pitch = a_scale_pitch ? a_scale_pitch : packed;
  m.w = w;
  m.w_scales = w_scales;
  m.y = y;
  return moe::hip_status(moe::launch_matmul_mx(m, as_stream(stream)));
}

}  // extern "C"
