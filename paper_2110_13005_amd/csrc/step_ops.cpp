// C entry points of the operations of a training step around the layer's own: scaled embedding, query / key norms with rotation,
// dropout, 8-bit linear maps.  They check their arguments and launch (embedding.hip, qk_norm.hip, dropout.hip, fp8.hip); nothing is
// allocated, nothing is kept between calls.
#include "../../include/axonn_stage.h"
#include "common.h"
#include "entry.h"

#include <cmath>

using namespace axonn;

namespace {

#define AX_TRY(expr)       \
  do {                     \
    int r_ = (expr);       \
    if (r_ != AXONN_OK) return r_; \
  } while (0)

int launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return AXONN_OK;
  return fail_entry(AXONN_EHIP, "%s: kernel launch failed: %s", what, hipGetErrorString(e));
}

// Rows that a launch's grid can hold (its threads in one dimension are counted in 32 bits).
constexpr int64_t kMaxRows = 1 << 24;

int embedding_sizes(const char* what, int64_t T, int64_t h, int64_t vocab) {
  if (T < 1 || h < 1 || vocab < 1) return fail_entry(AXONN_EINVAL, "%s: non-positive size", what);
  if (T > kMaxRows || h > 65535 || vocab > kMaxRows || vocab * h > (int64_t(1) << 34))
    return fail_entry(AXONN_EUNSUPPORTED, "%s: at most 2^24 tokens, h 65535, vocab 2^24 and vocab * h 2^34", what);
  return AXONN_OK;
}

int qk_shape(const char* what, int64_t T, int32_t seq_len, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
             int32_t rotary_dim, int32_t interleaved, float eps, const double* inv_freq, QkShape& q) {
  if (T < 1 || seq_len < 1 || n_heads < 1 || n_kv_heads < 1 || head_dim < 2) return fail_entry(AXONN_EINVAL, "%s: non-positive size", what);
  if (rotary_dim < 0 || rotary_dim > head_dim || rotary_dim % 2)
    return fail_entry(AXONN_EINVAL, "%s: rotary_dim must be even, 0 to head_dim", what);
  if (!(eps > 0.f) || !std::isfinite(eps)) return fail_entry(AXONN_EINVAL, "%s: eps must be positive and finite", what);
  if ((uintptr_t)inv_freq % 8) return fail_entry(AXONN_EINVAL, "%s: inv_freq must be 8-byte aligned", what);
  if (head_dim % 2 || head_dim > 256) return fail_entry(AXONN_EUNSUPPORTED, "%s: head dim must be even, at most 256", what);
  if (T > kMaxRows || n_heads > 4096 || n_kv_heads > 4096)
    return fail_entry(AXONN_EUNSUPPORTED, "%s: at most 2^24 tokens and 4096 heads of a kind", what);
  q = QkShape{T, seq_len, n_heads, n_kv_heads, head_dim, rotary_dim, interleaved != 0};
  return AXONN_OK;
}

int dropout(const char* what, int64_t T, int64_t h, const void* x, int64_t ld_x, const void* res, int64_t ld_res, float p,
            uint64_t seed, uint64_t offset, const uint64_t* offset_dev, void* out, int64_t ld_out, void* hip_stream) {
  if (!x || !out) return fail_entry(AXONN_EINVAL, "%s: null argument", what);
  if (T < 1 || h < 1) return fail_entry(AXONN_EINVAL, "%s: non-positive size", what);
  if (!(p >= 0.f && p <= 1.f)) return fail_entry(AXONN_EINVAL, "%s: p must be in [0, 1]", what);
  if (T > kMaxRows || h > kMaxRows || T * ((h + 7) / 8) > (int64_t(1) << 33))
    return fail_entry(AXONN_EUNSUPPORTED, "%s: at most 2^24 rows, 2^24 columns and 2^33 groups of 8 columns over all rows", what);
  if (ld_x < h || ld_out < h || (res && ld_res < h)) return fail_entry(AXONN_EINVAL, "%s: leading dimension too small", what);
  if ((out == x && ld_out != ld_x) || (out == res && ld_out != ld_res))
    return fail_entry(AXONN_EINVAL, "%s: in place with two leading dimensions", what);
  if ((uintptr_t)offset_dev % 8) return fail_entry(AXONN_EINVAL, "%s: offset_dev must be 8-byte aligned", what);
  LaunchTiming timing(PC_DROPOUT, (hipStream_t)hip_stream);
  return launched(launch_dropout(T, h, x, ld_x, res, ld_res, (uint32_t)std::lrint((double)p * 65536.0), seed, offset, offset_dev, out,
                                     ld_out, (hipStream_t)hip_stream), what);
}

}  // namespace

extern "C" {

int axonn_embedding_fwd(int64_t T, int64_t h, int64_t vocab, const int32_t* tokens, const void* table, float scale, void* out,
                        int64_t ld_out, void* hip_stream) {
  if (!tokens || !table || !out) return fail_entry(AXONN_EINVAL, "embedding_fwd: null argument");
  AX_TRY(embedding_sizes("embedding_fwd", T, h, vocab));
  if (ld_out < h) return fail_entry(AXONN_EINVAL, "embedding_fwd: ld_out < h");
  LaunchTiming timing(PC_EMBED, (hipStream_t)hip_stream);
  return launched(launch_embedding_fwd(T, h, vocab, tokens, table, scale, out, ld_out, (hipStream_t)hip_stream), "embedding_fwd");
}

int axonn_embedding_bwd_workspace(int64_t T, int64_t h, int64_t vocab, uint64_t* bytes) {
  if (!bytes) return fail_entry(AXONN_EINVAL, "embedding_bwd_workspace: null argument");
  AX_TRY(embedding_sizes("embedding_bwd_workspace", T, h, vocab));
  *bytes = embedding_bwd_ws_bytes(T, h, vocab);
  return AXONN_OK;
}

int axonn_embedding_bwd(int64_t T, int64_t h, int64_t vocab, const int32_t* tokens, const void* dout, int64_t ld_dout, float scale,
                        void* dtable, int32_t dtable_fp32, int32_t accumulate, void* workspace, void* hip_stream) {
  if (!tokens || !dout || !dtable || !workspace) return fail_entry(AXONN_EINVAL, "embedding_bwd: null argument");
  AX_TRY(embedding_sizes("embedding_bwd", T, h, vocab));
  if (ld_dout < h) return fail_entry(AXONN_EINVAL, "embedding_bwd: ld_dout < h");
  if ((uintptr_t)workspace % 16) return fail_entry(AXONN_EINVAL, "embedding_bwd: the workspace must be 16-byte aligned");
  if (dtable_fp32 && (uintptr_t)dtable % 4) return fail_entry(AXONN_EINVAL, "embedding_bwd: a 32-bit dtable must be 4-byte aligned");
  LaunchTiming timing(PC_EMBED, (hipStream_t)hip_stream);
  return launched(launch_embedding_bwd(T, h, vocab, tokens, dout, ld_dout, scale, dtable, dtable_fp32 != 0, accumulate != 0, workspace,
                  (hipStream_t)hip_stream), "embedding_bwd");
}

int axonn_qk_norm_rope_fwd(int64_t T, int32_t seq_len, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t rotary_dim,
                           int32_t interleaved, const void* qkv, int64_t ld_qkv, const void* gamma_q, const void* gamma_k, float eps,
                           const int32_t* positions, const double* inv_freq, void* out, int64_t ld_out, void* hip_stream) {
  if (!qkv || !gamma_q || !gamma_k || !out || (rotary_dim > 0 && !inv_freq)) return fail_entry(AXONN_EINVAL, "qk_norm_rope_fwd: null argument");
  QkShape q;
  AX_TRY(qk_shape("qk_norm_rope_fwd", T, seq_len, n_heads, n_kv_heads, head_dim, rotary_dim, interleaved, eps, inv_freq, q));
  const int64_t width = ((int64_t)n_heads + 2 * n_kv_heads) * head_dim;
  if (ld_qkv < width || ld_out < width) return fail_entry(AXONN_EINVAL, "qk_norm_rope_fwd: leading dimension too small");
  if (out == qkv && ld_out != ld_qkv) return fail_entry(AXONN_EINVAL, "qk_norm_rope_fwd: in place with two leading dimensions");
  LaunchTiming timing(PC_QK_NORM, (hipStream_t)hip_stream);
  return launched(launch_qk_norm_rope_fwd(q, qkv, ld_qkv, gamma_q, gamma_k, eps, positions, inv_freq, out, ld_out,
                  (hipStream_t)hip_stream), "qk_norm_rope_fwd");
}

int axonn_qk_norm_rope_bwd_workspace(int64_t T, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, uint64_t* bytes) {
  if (!bytes) return fail_entry(AXONN_EINVAL, "qk_norm_rope_bwd_workspace: null argument");
  QkShape q;
  AX_TRY(qk_shape("qk_norm_rope_bwd_workspace", T, 1, n_heads, n_kv_heads, head_dim, 0, 0, 1.f, nullptr, q));
  *bytes = qk_norm_rope_bwd_ws_bytes(T, head_dim);
  return AXONN_OK;
}

int axonn_qk_norm_rope_bwd(int64_t T, int32_t seq_len, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t rotary_dim,
                           int32_t interleaved, const void* dout, int64_t ld_dout, const void* qkv, int64_t ld_qkv, const void* gamma_q,
                           const void* gamma_k, float eps, const int32_t* positions, const double* inv_freq, void* dqkv, int64_t ld_dqkv,
                           float* dgamma_q, float* dgamma_k, void* workspace, void* hip_stream) {
  if (!dout || !qkv || !gamma_q || !gamma_k || !dqkv || !dgamma_q || !dgamma_k || !workspace || (rotary_dim > 0 && !inv_freq))
    return fail_entry(AXONN_EINVAL, "qk_norm_rope_bwd: null argument");
  QkShape q;
  AX_TRY(qk_shape("qk_norm_rope_bwd", T, seq_len, n_heads, n_kv_heads, head_dim, rotary_dim, interleaved, eps, inv_freq, q));
  const int64_t width = ((int64_t)n_heads + 2 * n_kv_heads) * head_dim;
  if (ld_dout < width || ld_qkv < width || ld_dqkv < width) return fail_entry(AXONN_EINVAL, "qk_norm_rope_bwd: leading dimension too small");
  if ((dqkv == dout && ld_dqkv != ld_dout) || (dqkv == qkv && ld_dqkv != ld_qkv))
    return fail_entry(AXONN_EINVAL, "qk_norm_rope_bwd: in place with two leading dimensions");
  if ((uintptr_t)workspace % 16) return fail_entry(AXONN_EINVAL, "qk_norm_rope_bwd: the workspace must be 16-byte aligned");
  LaunchTiming timing(PC_QK_NORM, (hipStream_t)hip_stream);
  return launched(launch_qk_norm_rope_bwd(q, dout, ld_dout, qkv, ld_qkv, gamma_q, gamma_k, eps, positions, inv_freq, dqkv, ld_dqkv,
                                              dgamma_q, dgamma_k, (float*)workspace, (hipStream_t)hip_stream), "qk_norm_rope_bwd");
}

int axonn_dropout_fwd(int64_t T, int64_t h, const void* x, int64_t ld_x, const void* res, int64_t ld_res, float p, uint64_t seed,
                      uint64_t offset, const uint64_t* offset_dev, void* out, int64_t ld_out, void* hip_stream) {
  return dropout("dropout_fwd", T, h, x, ld_x, res, ld_res, p, seed, offset, offset_dev, out, ld_out, hip_stream);
}
int axonn_dropout_bwd(int64_t T, int64_t h, const void* dout, int64_t ld_dout, float p, uint64_t seed, uint64_t offset,
                      const uint64_t* offset_dev, void* dx, int64_t ld_dx, void* hip_stream) {
  return dropout("dropout_bwd", T, h, dout, ld_dout, nullptr, 0, p, seed, offset, offset_dev, dx, ld_dx, hip_stream);
}

int axonn_fp8_quantize(int64_t R, int64_t C, const void* x, int64_t ld_x, void* q, uint8_t* scale, void* q_t, uint8_t* scale_t,
                       void* hip_stream) {
  if (!x) return fail_entry(AXONN_EINVAL, "fp8_quantize: null argument");
  if ((q == nullptr) != (scale == nullptr) || (q_t == nullptr) != (scale_t == nullptr) || (!q && !q_t))
    return fail_entry(AXONN_EINVAL, "fp8_quantize: codes and scales of one form at least, each with the other");
  if (R < 1 || C < 1) return fail_entry(AXONN_EINVAL, "fp8_quantize: non-positive size");
  if (R > (1 << 22) || C > (1 << 22) || R * C > (int64_t(1) << 35))
    return fail_entry(AXONN_EUNSUPPORTED, "fp8_quantize: dimension above 2^22 or more than 2^35 elements");
  if (ld_x < C) return fail_entry(AXONN_EINVAL, "fp8_quantize: ld_x < C");
  if ((uintptr_t)q % 16 || (uintptr_t)q_t % 16 || (uintptr_t)scale % 4 || (uintptr_t)scale_t % 4)
    return fail_entry(AXONN_EINVAL, "fp8_quantize: codes must be 16-byte aligned, scales 4-byte aligned");
  LaunchTiming timing(PC_FP8_QUANT, (hipStream_t)hip_stream);
  return launched(launch_fp8_quantize(R, C, x, ld_x, q, scale, q_t, scale_t, (hipStream_t)hip_stream), "fp8_quantize");
}

int axonn_gemm_fp8(int32_t epilogue, int64_t M, int64_t N, int64_t K, const void* A, const uint8_t* a_scale, const void* B,
                   const uint8_t* b_scale, void* C, int64_t ldc, const void* bias, const void* res, int64_t ld_res, void* aux,
                   int64_t ld_aux, int32_t accumulate, void* hip_stream) {
  if (!A || !a_scale || !B || !b_scale || !C) return fail_entry(AXONN_EINVAL, "gemm_fp8: null operand");
  if (M < 1 || N < 1 || K < 1) return fail_entry(AXONN_EINVAL, "gemm_fp8: non-positive size");
  if (epilogue < 0 || epilogue > 5) return fail_entry(AXONN_EINVAL, "gemm_fp8: unknown epilogue %d", epilogue);
  if (M > (1 << 22) || N > (1 << 22) || K > (1 << 22) || M * N > (int64_t(1) << 38))
    return fail_entry(AXONN_EUNSUPPORTED, "gemm_fp8: dimension above 2^22 or more than 2^38 results");
  if (ldc < N) return fail_entry(AXONN_EINVAL, "gemm_fp8: leading dimension too small");
  if (epilogue == EPI_BIAS_RES && (!res || ld_res < N)) return fail_entry(AXONN_EINVAL, "gemm_fp8: epilogue 1 needs res with ld_res >= N");
  if ((epilogue == EPI_BIAS_GELU || epilogue == EPI_DGELU) && (!aux || ld_aux < N))
    return fail_entry(AXONN_EINVAL, "gemm_fp8: epilogue %d needs aux with ld_aux >= N", epilogue);
  if ((epilogue == EPI_BIAS_RES && C == res && ldc != ld_res) || (epilogue == EPI_DGELU && C == aux && ldc != ld_aux))
    return fail_entry(AXONN_EINVAL, "gemm_fp8: in place with two leading dimensions");
  if (epilogue == EPI_BIAS_GELU && C == aux) return fail_entry(AXONN_EINVAL, "gemm_fp8: two results in one place");
  if ((uintptr_t)A % 16 || (uintptr_t)B % 16 || (uintptr_t)a_scale % 4 || (uintptr_t)b_scale % 4)
    return fail_entry(AXONN_EINVAL, "gemm_fp8: codes must be 16-byte aligned, scales 4-byte aligned");
  if (epilogue == EPI_ACC_F32 && (uintptr_t)C % 4) return fail_entry(AXONN_EINVAL, "gemm_fp8: a 32-bit result must be 4-byte aligned");
  LaunchTiming timing(PC_GEMM_FP8, (hipStream_t)hip_stream);
  return launched(launch_gemm_fp8(epilogue, M, N, K, A, a_scale, B, b_scale, C, ldc, bias, res, ld_res, aux, ld_aux, accumulate,
                  (hipStream_t)hip_stream), "gemm_fp8");
}

}  // extern "C"
