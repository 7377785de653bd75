// C-ABI layer of the losses on logits: argument checks; everything else is enqueued.
#include "logits_checks.h"

using namespace lb;

namespace {

size_t workspace_of(const lbfgsb_logits* l, bool grad) {
    if (l->rows == 0 || row_splits(l->rows, l->vocab, (int)size_of(l->dtype), grad) == 1) return 0;
    return (l->rows * sizeof(SplitRow) + 255) & ~(size_t)255;
}

int check_workspace(const lbfgsb_logits* l, bool grad, const void* ws, size_t bytes) {
    return check_space(workspace_of(l, grad), ws, bytes);
}

LogitsArgs args_of(const lbfgsb_logits* l, bool grad) {
    const double s = 1.0 / l->temperature;
    return {l->z, grad ? l->grad : nullptr, l->rows, l->ld, l->ld_grad, (int)l->vocab, s, factor_of(s)};
}

int check_scale(double scale, const float* loss) {
    if (!std::isfinite(scale)) return fail(LBFGSB_E_INVALID_ARG, "scale is not finite");
    if (!loss) return fail(LBFGSB_E_INVALID_ARG, "loss is NULL");
    return LBFGSB_OK;
}

}  // namespace

extern "C" {

size_t lbfgsb_logits_workspace_bytes(const lbfgsb_logits* logits_host) {
    if (check_shape(logits_host)) return 0;
    return workspace_of(logits_host, logits_host->grad != nullptr);
}

int lbfgsb_token_logprob(const lbfgsb_logits* logits_host, const int64_t* labels, float* logp, float* lse, float* lse_rest,
                         float* entropy, void* workspace, size_t workspace_bytes, void* hip_stream) {
    return lbfgsb_token_logprob_stats(logits_host, labels, logp, lse, lse_rest, entropy, nullptr, nullptr, workspace, workspace_bytes, hip_stream);
}

int lbfgsb_token_logprob_stats(const lbfgsb_logits* logits_host, const int64_t* labels, float* logp, float* lse, float* lse_rest,
                               float* entropy, float* top, float* sum, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (int rc = check_logits(logits_host, -1)) return rc;
    if (int rc = check_workspace(logits_host, false, workspace, workspace_bytes)) return rc;
    if (logits_host->rows == 0) return LBFGSB_OK;
    if (!labels || !logp || !lse) return fail(LBFGSB_E_INVALID_ARG, "labels, logp and lse must not be NULL");
    if (!top != !sum) return fail(LBFGSB_E_INVALID_ARG, "top goes with sum");
    HIP_TRY(launch_token_logprob(args_of(logits_host, false), logits_host->dtype, {labels, logp, lse, lse_rest, entropy, top, sum},
                                 (SplitRow*)workspace, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

int lbfgsb_token_logprob_grad(const lbfgsb_logits* logits_host, const int64_t* labels, const float* lse, const float* lse_rest,
                              const float* entropy, const float* d_logp, const float* d_entropy, void* hip_stream) {
    if (int rc = check_logits(logits_host, 1)) return rc;
    if (logits_host->rows == 0) return LBFGSB_OK;
    if (!labels || !lse || !d_logp) return fail(LBFGSB_E_INVALID_ARG, "labels, lse and d_logp must not be NULL");
    if (d_entropy && !entropy) return fail(LBFGSB_E_INVALID_ARG, "d_entropy goes with the entropy");
    HIP_TRY(launch_token_logprob_grad(args_of(logits_host, true), logits_host->dtype,
                                      {labels, nullptr, nullptr, lse, lse_rest, entropy, d_logp, d_entropy, logits_host->temperature}, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

int lbfgsb_token_logprob_stats_grad(const lbfgsb_logits* logits_host, const int64_t* labels, const float* top, const float* sum,
                                    const float* entropy, const float* d_logp, const float* d_entropy, void* hip_stream) {
    if (int rc = check_logits(logits_host, 1)) return rc;
    if (logits_host->rows == 0) return LBFGSB_OK;
    if (!labels || !top || !sum || !d_logp) return fail(LBFGSB_E_INVALID_ARG, "labels, top, sum and d_logp must not be NULL");
    if (d_entropy && !entropy) return fail(LBFGSB_E_INVALID_ARG, "d_entropy goes with the entropy");
    HIP_TRY(launch_token_logprob_grad(args_of(logits_host, true), logits_host->dtype,
                                      {labels, top, sum, nullptr, nullptr, entropy, d_logp, d_entropy, logits_host->temperature}, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

int lbfgsb_distill_loss(const lbfgsb_logits* logits_host, const lbfgsb_teacher* teacher_host, const float* weight, double scale,
                        float* loss, float* row_loss, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (int rc = check_logits(logits_host, 0)) return rc;
    if (int rc = check_workspace(logits_host, logits_host->grad != nullptr, workspace, workspace_bytes)) return rc;
    const lbfgsb_teacher* t = teacher_host;
    if (!t) return fail(LBFGSB_E_INVALID_ARG, "teacher is NULL");
    if (logits_host->vocab > kMaxDistillVocab) return fail(LBFGSB_E_INVALID_ARG, "distillation takes a vocabulary of at most 2^19");
    if (t->index_type != LBFGSB_I32 && t->index_type != LBFGSB_I64) return fail(LBFGSB_E_INVALID_ARG, "unknown index type %d", t->index_type);
    if (!is_logit_type(t->logit_type)) return fail(LBFGSB_E_INVALID_ARG, "teacher: unknown logit type %d", t->logit_type);
    if (t->top < 1 || t->top > kMaxTop) return fail(LBFGSB_E_INVALID_ARG, "top must be in 1..%d (got %lld)", kMaxTop, (long long)t->top);
    if (t->ld < t->top || t->ld > kMaxLd) return fail(LBFGSB_E_INVALID_ARG, "teacher: ld must be in top..2^31 (got %lld)", (long long)t->ld);
    if (int rc = check_scale(scale, loss)) return rc;
    if (logits_host->rows && (!t->index || !t->logit || !row_loss || misaligned(t->index, t->index_type == LBFGSB_I32 ? 4 : 8) ||
                              misaligned(t->logit, size_of(t->logit_type))))
        return fail(LBFGSB_E_INVALID_ARG, "index, logit or row_loss is NULL or not aligned to its elements");
    HIP_TRY(launch_distill(args_of(logits_host, true), logits_host->dtype,
                           {t->index, t->logit, t->lse, weight, row_loss, t->ld, (int)t->top, t->index_type, t->logit_type, scale}, loss,
                           (SplitRow*)workspace, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

int lbfgsb_policy_loss(const lbfgsb_logits* logits_host, const lbfgsb_rollout* rollout_host, const lbfgsb_policy_options* opt_host,
                       double scale, float* loss, float* row_loss, float* logp, float* entropy, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
    if (int rc = check_logits(logits_host, 0)) return rc;
    if (int rc = check_workspace(logits_host, logits_host->grad != nullptr, workspace, workspace_bytes)) return rc;
    const lbfgsb_rollout* p = rollout_host;
    const lbfgsb_policy_options* o = opt_host;
    if (!p || !o) return fail(LBFGSB_E_INVALID_ARG, "rollout or options is NULL");
    if (!(o->clip_low >= 0.0 && o->clip_low <= 1.0) || !(o->clip_high >= 0.0) || !std::isfinite(o->kl_coef) || !std::isfinite(o->entropy_coef))
        return fail(LBFGSB_E_INVALID_ARG, "bad option value");
    if (o->kl_kind < LBFGSB_KL_1 || o->kl_kind > LBFGSB_KL_3) return fail(LBFGSB_E_INVALID_ARG, "unknown kl_kind %d", o->kl_kind);
    if (int rc = check_scale(scale, loss)) return rc;
    if (logits_host->rows) {
        if (!p->labels || !p->old_logp || !p->advantage || !row_loss || !logp)
            return fail(LBFGSB_E_INVALID_ARG, "labels, old_logp, advantage, row_loss and logp must not be NULL");
        if (o->kl_coef != 0.0 && !p->ref_logp) return fail(LBFGSB_E_INVALID_ARG, "kl_coef goes with ref_logp");
    }
    HIP_TRY(launch_policy(args_of(logits_host, true), logits_host->dtype,
                          {p->labels, p->old_logp, p->advantage, p->ref_logp, p->weight, row_loss, logp, entropy, (float)(1.0 - o->clip_low),
                           (float)(1.0 + o->clip_high), (float)o->kl_coef, (float)o->entropy_coef, o->kl_kind, scale},
                          loss, (SplitRow*)workspace, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

int lbfgsb_preference_loss(int64_t tokens, int64_t pairs, const float* logp, const float* ref_logp, const int64_t* offsets,
                           const uint8_t* mask, const float* weight, const lbfgsb_preference_options* opt_host, double scale,
                           float* loss, float* pair_loss, float* rewards, float* grad, void* hip_stream) {
    const lbfgsb_preference_options* o = opt_host;
    if (tokens < 0 || tokens > (1ll << 40) || pairs < 0 || pairs > kMaxRows / 2)
        return fail(LBFGSB_E_INVALID_ARG, "tokens must be in 0..2^40 and pairs in 0..2^30-1 (got %lld, %lld)", (long long)tokens, (long long)pairs);
    if (!o) return fail(LBFGSB_E_INVALID_ARG, "options is NULL");
    if (o->kind < LBFGSB_PAIR_SIGMOID || o->kind > LBFGSB_PAIR_IPO) return fail(LBFGSB_E_INVALID_ARG, "unknown kind %d", o->kind);
    if (!(o->beta > 0.0) || !std::isfinite(o->beta) || !std::isfinite(1.0 / o->beta) || !std::isfinite(o->margin) ||
        !(o->label_smoothing >= 0.0 && o->label_smoothing < 1.0) || (o->label_smoothing != 0.0 && o->kind != LBFGSB_PAIR_SIGMOID))
        return fail(LBFGSB_E_INVALID_ARG, "bad option value");
    if (int rc = check_scale(scale, loss)) return rc;
    if (pairs > 0 && (!offsets || !pair_loss || !rewards)) return fail(LBFGSB_E_INVALID_ARG, "offsets, pair_loss and rewards must not be NULL");
    if (pairs > 0 && tokens > 0 && !logp) return fail(LBFGSB_E_INVALID_ARG, "logp is NULL");
    HIP_TRY(launch_preference({tokens, pairs, logp, ref_logp, weight, offsets, mask, pair_loss, rewards, grad, o->beta, o->label_smoothing,
                               o->margin, scale, o->kind, o->length_normalised},
                              loss, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

}  // extern "C"
