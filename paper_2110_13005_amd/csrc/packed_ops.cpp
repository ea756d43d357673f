// C entry points of the operations on packed sequences: attention inside sequences of different lengths, and the losses that a training
// step on them ends in.  They check their arguments and launch (attention_packed.hip, losses.hip); nothing is allocated, nothing is
// kept between calls.
#include "entry.h"

#include <cmath>

using namespace axonn;

namespace {

// Sizes that the launches' grids hold (their threads in one dimension are counted in 32 bits); the rows of a tile that a descriptor's
// 32-bit offsets reach.
constexpr int64_t kMaxTokens = 1 << 24, kMaxSequences = 1 << 20, kMaxLd = 1 << 22;

int packed_sequences(const char* what, int64_t T, int32_t n_seq) {
  if (T < 1 || n_seq < 1) return fail_entry(AXONN_EINVAL, "%s: non-positive size", what);
  if (T > kMaxTokens || n_seq > kMaxSequences) return fail_entry(AXONN_EUNSUPPORTED, "%s: at most 2^24 rows and 2^20 sequences", what);
  return AXONN_OK;
}

int packed_shape(const char* what, int64_t T, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                 PackedShape& s) {
  AX_TRY(packed_sequences(what, T, n_seq));
  if (n_heads < 1 || n_kv_heads < 1 || head_dim < 1) return fail_entry(AXONN_EINVAL, "%s: non-positive size", what);
  if (n_heads % n_kv_heads) return fail_entry(AXONN_EINVAL, "%s: n_heads must be a multiple of n_kv_heads", what);
  if (!(scale > 0.f) || !std::isfinite(scale)) return fail_entry(AXONN_EINVAL, "%s: scale must be positive and finite", what);
  if (head_dim % 4 || head_dim > 192) return fail_entry(AXONN_EUNSUPPORTED, "%s: head dim must be a multiple of 4, at most 192", what);
  if (n_heads > 4096 || T * n_heads > (1 << 27) || (int64_t)n_seq * n_heads > (1 << 22))
    return fail_entry(AXONN_EUNSUPPORTED, "%s: at most 4096 heads, 2^27 rows and 2^22 sequences times heads", what);
  s = PackedShape{T, n_seq, n_heads, n_kv_heads, head_dim, scale};
  return AXONN_OK;
}
int packed_ld(const char* what, int64_t width, int64_t ld) {
  if (ld < width) return fail_entry(AXONN_EINVAL, "%s: leading dimension too small", what);
  if (ld > kMaxLd) return fail_entry(AXONN_EUNSUPPORTED, "%s: leading dimensions of at most 2^22", what);
  return AXONN_OK;
}

int logits_shape(const char* what, int64_t T, int64_t V, int64_t ld) {
  if (T < 1 || V < 1) return fail_entry(AXONN_EINVAL, "%s: non-positive size", what);
  if (T > (1 << 21) || V > (1 << 20) || T * V > (int64_t(1) << 36))
    return fail_entry(AXONN_EUNSUPPORTED, "%s: at most 2^21 rows, a vocabulary of 2^20 and 2^36 logits", what);
  if (ld < V) return fail_entry(AXONN_EINVAL, "%s: ld_logits < V", what);
  return AXONN_OK;
}
int logits_gradient(const char* what, int64_t V, const void* logits, int64_t ld, const void* dlogits, int64_t ld_d, float loss_scale) {
  if (!(loss_scale > 0.f) || !std::isfinite(loss_scale)) return fail_entry(AXONN_EINVAL, "%s: loss_scale must be positive and finite", what);
  if (!dlogits) return AXONN_OK;
  if (ld_d < V) return fail_entry(AXONN_EINVAL, "%s: ld_dlogits < V", what);
  if (dlogits == logits && ld_d != ld) return fail_entry(AXONN_EINVAL, "%s: in place with two leading dimensions", what);
  return AXONN_OK;
}

}  // namespace

extern "C" {

int axonn_attention_packed_plan_bytes(int64_t T, int32_t n_seq, uint64_t* bytes) {
  if (!bytes) return fail_entry(AXONN_EINVAL, "attention_packed_plan_bytes: null argument");
  AX_TRY(packed_sequences("attention_packed_plan_bytes", T, n_seq));
  *bytes = attention_packed_plan_size(T, n_seq);
  return AXONN_OK;
}

int axonn_attention_packed_plan(int64_t T, int32_t n_seq, const int32_t* offsets, void* plan, void* hip_stream) {
  if (!offsets || !plan) return fail_entry(AXONN_EINVAL, "attention_packed_plan: null argument");
  AX_TRY(packed_sequences("attention_packed_plan", T, n_seq));
  if ((uintptr_t)plan % 16) return fail_entry(AXONN_EINVAL, "attention_packed_plan: the plan must be 16-byte aligned");
  LaunchTiming timing(PC_ATTN_FWD, (hipStream_t)hip_stream);
  return launched(launch_attention_packed_plan(T, n_seq, offsets, plan, (hipStream_t)hip_stream), "attention_packed_plan");
}

int axonn_attention_packed_fwd(int64_t T, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                               const void* plan, const void* qkv, int64_t ld_qkv, void* o, int64_t ld_o, float* lse, void* hip_stream) {
  const char* what = "attention_packed_fwd";
  if (!plan || !qkv || !o || !lse) return fail_entry(AXONN_EINVAL, "%s: null argument", what);
  PackedShape s;
  AX_TRY(packed_shape(what, T, n_seq, n_heads, n_kv_heads, head_dim, scale, s));
  AX_TRY(packed_ld(what, ((int64_t)n_heads + 2 * n_kv_heads) * head_dim, ld_qkv));
  AX_TRY(packed_ld(what, (int64_t)n_heads * head_dim, ld_o));
  if ((uintptr_t)plan % 16 || (uintptr_t)lse % 4) return fail_entry(AXONN_EINVAL, "%s: the plan must be 16-byte aligned, lse 4-byte aligned", what);
  if (o == qkv) return fail_entry(AXONN_EINVAL, "%s: o may not be qkv", what);
  LaunchTiming timing(PC_ATTN_FWD, (hipStream_t)hip_stream);
  return launched(launch_attention_packed_fwd(s, plan, qkv, ld_qkv, o, ld_o, lse, (hipStream_t)hip_stream), what);
}

int axonn_attention_packed_bwd_workspace(int64_t T, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, uint64_t* bytes) {
  if (!bytes) return fail_entry(AXONN_EINVAL, "attention_packed_bwd_workspace: null argument");
  PackedShape s;
  AX_TRY(packed_shape("attention_packed_bwd_workspace", T, n_seq, n_heads, n_kv_heads, head_dim, 1.f, s));
  *bytes = attention_packed_bwd_ws_bytes(s);
  return AXONN_OK;
}

int axonn_attention_packed_bwd(int64_t T, int32_t n_seq, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                               const void* plan, const void* qkv, int64_t ld_qkv, const void* o, int64_t ld_o, const float* lse,
                               const void* dout, int64_t ld_dout, void* dqkv, int64_t ld_dqkv, void* workspace, void* hip_stream) {
  const char* what = "attention_packed_bwd";
  if (!plan || !qkv || !o || !lse || !dout || !dqkv || !workspace) return fail_entry(AXONN_EINVAL, "%s: null argument", what);
  PackedShape s;
  AX_TRY(packed_shape(what, T, n_seq, n_heads, n_kv_heads, head_dim, scale, s));
  const int64_t width = ((int64_t)n_heads + 2 * n_kv_heads) * head_dim, width_o = (int64_t)n_heads * head_dim;
  AX_TRY(packed_ld(what, width, ld_qkv));
  AX_TRY(packed_ld(what, width_o, ld_o));
  AX_TRY(packed_ld(what, width_o, ld_dout));
  AX_TRY(packed_ld(what, width, ld_dqkv));
  if ((uintptr_t)plan % 16 || (uintptr_t)workspace % 16 || (uintptr_t)lse % 4)
    return fail_entry(AXONN_EINVAL, "%s: the plan and the workspace must be 16-byte aligned, lse 4-byte aligned", what);
  if (dqkv == qkv || dqkv == o || dqkv == dout) return fail_entry(AXONN_EINVAL, "%s: dqkv may not be an operand", what);
  LaunchTiming timing(PC_ATTN_BWD, (hipStream_t)hip_stream);
  return launched(launch_attention_packed_bwd(s, plan, qkv, ld_qkv, o, ld_o, lse, dout, ld_dout, dqkv, ld_dqkv, workspace,
                                              (hipStream_t)hip_stream), what);
}

int axonn_token_logprobs_fwd(int64_t T, int64_t V, const void* logits, int64_t ld_logits, const int32_t* targets, float* logp, float* lse,
                             void* hip_stream) {
  if (!logits || !targets || !logp || !lse) return fail_entry(AXONN_EINVAL, "token_logprobs_fwd: null argument");
  AX_TRY(logits_shape("token_logprobs_fwd", T, V, ld_logits));
  LaunchTiming timing(PC_LOSSES, (hipStream_t)hip_stream);
  return launched(launch_token_logprobs_fwd(T, V, logits, ld_logits, targets, logp, lse, (hipStream_t)hip_stream), "token_logprobs_fwd");
}

int axonn_token_logprobs_bwd(int64_t T, int64_t V, const void* logits, int64_t ld_logits, const int32_t* targets, const float* lse,
                             const float* dlogp, void* dlogits, int64_t ld_dlogits, void* hip_stream) {
  if (!logits || !targets || !lse || !dlogp || !dlogits) return fail_entry(AXONN_EINVAL, "token_logprobs_bwd: null argument");
  AX_TRY(logits_shape("token_logprobs_bwd", T, V, ld_logits));
  AX_TRY(logits_gradient("token_logprobs_bwd", V, logits, ld_logits, dlogits, ld_dlogits, 1.f));
  LaunchTiming timing(PC_LOSSES, (hipStream_t)hip_stream);
  return launched(launch_token_logprobs_bwd(T, V, logits, ld_logits, targets, lse, dlogp, dlogits, ld_dlogits, (hipStream_t)hip_stream),
                  "token_logprobs_bwd");
}

int axonn_policy_loss(int64_t T, int64_t V, const void* logits, int64_t ld_logits, const int32_t* targets, const float* old_logp,
                      const float* ref_logp, const float* advantage, const float* weight, float clip_low, float clip_high, float kl_coef,
                      float loss_scale, float* logp, float* token_loss, float* loss, void* dlogits, int64_t ld_dlogits, void* hip_stream) {
  const char* what = "policy_loss";
  if (!logits || !targets || !old_logp || !advantage || !weight || !token_loss) return fail_entry(AXONN_EINVAL, "%s: null argument", what);
  AX_TRY(logits_shape(what, T, V, ld_logits));
  AX_TRY(logits_gradient(what, V, logits, ld_logits, dlogits, ld_dlogits, loss_scale));
  if (!(clip_low >= 0.f && clip_low <= 1.f) || !(clip_high >= 0.f) || !std::isfinite(clip_high))
    return fail_entry(AXONN_EINVAL, "%s: clip_low must be in [0, 1], clip_high at least 0 and finite", what);
  if (!(kl_coef >= 0.f) || !std::isfinite(kl_coef)) return fail_entry(AXONN_EINVAL, "%s: kl_coef must be at least 0 and finite", what);
  if (kl_coef > 0.f && !ref_logp) return fail_entry(AXONN_EINVAL, "%s: a KL term needs ref_logp", what);
  const PolicyArgs p{(int)V, logits, ld_logits, targets, old_logp, kl_coef > 0.f ? ref_logp : nullptr, advantage, weight,
                     (float)(1.0 - clip_low), (float)(1.0 + clip_high), kl_coef, loss_scale, logp, token_loss, dlogits, ld_dlogits};
  LaunchTiming timing(PC_LOSSES, (hipStream_t)hip_stream);
  return launched(launch_policy_loss(T, p, loss, (hipStream_t)hip_stream), what);
}

int axonn_preference_loss(int64_t T, int32_t n_pairs, int64_t V, const int32_t* offsets, const int32_t* targets, const float* logp,
                          const float* ref_logp, float beta, float label_smoothing, float scale, float loss_scale, float* pair_loss,
                          float* loss, float* dlogp, void* hip_stream) {
  const char* what = "preference_loss";
  if (!offsets || !targets || !logp || !pair_loss || !dlogp) return fail_entry(AXONN_EINVAL, "%s: null argument", what);
  if (n_pairs < 1) return fail_entry(AXONN_EINVAL, "%s: non-positive size", what);
  if (n_pairs > kMaxSequences / 2) return fail_entry(AXONN_EUNSUPPORTED, "%s: at most 2^19 pairs", what);
  AX_TRY(logits_shape(what, T, V, V));
  if (!(beta > 0.f) || !std::isfinite(beta) || !(scale > 0.f) || !std::isfinite(scale) || !(loss_scale > 0.f) || !std::isfinite(loss_scale))
    return fail_entry(AXONN_EINVAL, "%s: beta, scale and loss_scale must be positive and finite", what);
  if (!(label_smoothing >= 0.f && label_smoothing <= 1.f)) return fail_entry(AXONN_EINVAL, "%s: label_smoothing must be in [0, 1]", what);
  const PreferenceArgs p{(int)T, n_pairs, (int)V, offsets, targets, logp, ref_logp, beta, label_smoothing, scale, loss_scale, pair_loss, dlogp};
  LaunchTiming timing(PC_LOSSES, (hipStream_t)hip_stream);
  return launched(launch_preference_loss(p, loss, (hipStream_t)hip_stream), what);
}

int axonn_distill_loss(int64_t T, int64_t V, int32_t K, const void* logits, int64_t ld_logits, const float* teacher_logits,
                       const int32_t* teacher_ids, int64_t ld_teacher, const float* teacher_lse, float temperature, const float* weight,
                       float loss_scale, float* token_loss, float* loss, void* dlogits, int64_t ld_dlogits, void* hip_stream) {
  const char* what = "distill_loss";
  if (!logits || !teacher_logits || !teacher_ids || !weight || !token_loss) return fail_entry(AXONN_EINVAL, "%s: null argument", what);
  AX_TRY(logits_shape(what, T, V, ld_logits));
  AX_TRY(logits_gradient(what, V, logits, ld_logits, dlogits, ld_dlogits, loss_scale));
  if (K < 1) return fail_entry(AXONN_EINVAL, "%s: non-positive size", what);
  if (K > kDistillMax || V > kDistillMaxVocab)
    return fail_entry(AXONN_EUNSUPPORTED, "%s: at most %d entries per token and a vocabulary of %d", what, kDistillMax, kDistillMaxVocab);
  if (ld_teacher < K) return fail_entry(AXONN_EINVAL, "%s: ld_teacher < K", what);
  if (!(temperature >= 0x1p-16f && temperature <= 0x1p16f))
    return fail_entry(AXONN_EINVAL, "%s: temperature must be in [2^-16, 2^16]", what);
  const DistillArgs a{(int)V, K, logits, ld_logits, teacher_logits, teacher_ids, ld_teacher, teacher_lse, weight, temperature,
                      (float)(1.4426950408889634 / temperature), loss_scale, token_loss, dlogits, ld_dlogits};
  LaunchTiming timing(PC_LOSSES, (hipStream_t)hip_stream);
  return launched(launch_distill_loss(T, a, loss, (hipStream_t)hip_stream), what);
}

}  // extern "C"
