// C-ABI layer of what makes rollouts: argument checks; everything else is enqueued.
#include "draws.h"
#include "logits_checks.h"
#include "weights4.h"

using namespace lb;

namespace {

constexpr int64_t kMaxWeightRows = 1 << 28, kMaxWeightCols = 1 << 24, kMaxWeights = 1ll << 35;

int check_weights(const lbfgsb_weights4* w) {
    if (!w) return fail(LBFGSB_E_INVALID_ARG, "weights is NULL");
    if (w->rows < 1 || w->rows > kMaxWeightRows || w->cols < 1 || w->cols > kMaxWeightCols)
        return fail(LBFGSB_E_INVALID_ARG, "weights: rows must be in 1..2^28 and cols in 1..2^24 (got %lld, %lld)", (long long)w->rows, (long long)w->cols);
    if (((w->rows + 63) & ~63ll) * ((w->cols + 127) & ~127ll) > kMaxWeights) return fail(LBFGSB_E_INVALID_ARG, "weights: more than 2^35 entries");
    if (w->group < 32 || w->group > kMaxWeightCols || (w->group & (w->group - 1)))
        return fail(LBFGSB_E_INVALID_ARG, "group must be a power of two in 32..2^24 (got %lld)", (long long)w->group);
    if (!is_logit_type(w->scale_type)) return fail(LBFGSB_E_INVALID_ARG, "weights: unknown scale type %d", w->scale_type);
    return LBFGSB_OK;
}

Packed4 packed_of(const lbfgsb_weights4* w) {
    int l = 5;
    while ((1ll << l) < w->group) ++l;
    return {w->rows, (int)w->cols, l, w->scale_type, w->zero ? 1 : 0};
}

int check_plain(const lbfgsb_weights4* w) {
    const size_t b = size_of(w->scale_type);
    if (!w->codes || !w->scale || misaligned(w->scale, b) || misaligned(w->zero, b))
        return fail(LBFGSB_E_INVALID_ARG, "codes or scale is NULL, or scale or zero not aligned to its elements");
    return LBFGSB_OK;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

int check_drafts(const lbfgsb_drafts* d) {
    if (!d) return fail(LBFGSB_E_INVALID_ARG, "drafts is NULL");
    if (!is_logit_type(d->dtype)) return fail(LBFGSB_E_INVALID_ARG, "logits: unknown dtype %d", d->dtype);
    if (d->drafts < 0 || d->drafts > kMaxDrafts || d->requests < 0 || d->requests > kMaxRows || d->requests * (d->drafts + 1) > kMaxRows)
        return fail(LBFGSB_E_INVALID_ARG, "drafts must be in 0..128 and requests * (drafts + 1) in 0..2^31-1 (got %lld, %lld)", (long long)d->drafts,
                    (long long)d->requests);
    if (d->vocab < 1 || d->vocab > kMaxDrawVocab) return fail(LBFGSB_E_INVALID_ARG, "vocab must be in 1..2^21 (got %lld)", (long long)d->vocab);
    return LBFGSB_OK;
}

int check_strides(const lbfgsb_drafts* d, int64_t ld, int64_t ld_request, int64_t positions, const char* name) {
    if ((positions > 1 && (ld < d->vocab || ld > kMaxLd * 128)) || (d->requests > 1 && (ld_request < d->vocab || ld_request > kMaxLd * 128)))
        return fail(LBFGSB_E_INVALID_ARG, "%s: strides must be in vocab..2^38 (got %lld, %lld)", name, (long long)ld, (long long)ld_request);
    return LBFGSB_OK;
}

VerifySpace space_of(const lbfgsb_drafts* d) {
    const bool drafter = d->draft_z && d->drafts > 0;
    return verify_space(d->requests, d->drafts, d->vocab, (int)size_of(d->dtype), drafter, drafter && !d->draft_logp);
}

}  // namespace

extern "C" {

int lbfgsb_quantize4(int dtype, int64_t ld, const void* w, const lbfgsb_weights4* to_host, void* hip_stream) {
    if (int rc = check_weights(to_host)) return rc;
    if (!is_logit_type(dtype)) return fail(LBFGSB_E_INVALID_ARG, "w: unknown dtype %d", dtype);
    if (ld < to_host->cols || ld > kMaxLd) return fail(LBFGSB_E_INVALID_ARG, "ld must be in cols..2^31 (got %lld)", (long long)ld);
    if (!w || misaligned(w, size_of(dtype))) return fail(LBFGSB_E_INVALID_ARG, "w is NULL or not aligned to its elements");
    if (int rc = check_plain(to_host)) return rc;
    HIP_TRY(launch_quantize4(dtype, ld, w, to_host->rows, to_host->cols, to_host->group, to_host->scale_type, (uint8_t*)to_host->codes,
                             (void*)to_host->scale, (void*)to_host->zero, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

size_t lbfgsb_packed4_bytes(const lbfgsb_weights4* weights_host) {
    return check_weights(weights_host) ? 0 : packed_of(weights_host).bytes();
}

int lbfgsb_pack4(const lbfgsb_weights4* weights_host, void* packed, size_t packed_bytes, void* hip_stream) {
    if (int rc = check_weights(weights_host)) return rc;
    if (int rc = check_plain(weights_host)) return rc;
    const Packed4 p = packed_of(weights_host);
    if (!packed || misaligned(packed, 16)) return fail(LBFGSB_E_INVALID_ARG, "packed is NULL or not aligned to 16 bytes");
    if (packed_bytes < p.bytes()) return fail(LBFGSB_E_INVALID_ARG, "packed too small: %zu bytes, need %zu", packed_bytes, p.bytes());
    HIP_TRY(launch_pack4(p, weights_host->codes, weights_host->scale, weights_host->zero, packed, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

size_t lbfgsb_matvec4_workspace_bytes(const lbfgsb_weights4* weights_host, int64_t tokens, int x_type) {
    if (check_weights(weights_host) || tokens < 1 || tokens > kMaxRows || !is_logit_type(x_type)) return 0;
    return matvec4_bytes(packed_of(weights_host), tokens, x_type);
}

int lbfgsb_matvec4(const lbfgsb_weights4* weights_host, const void* packed, int64_t tokens, int x_type, int64_t ld_x, const void* x, int y_type,
                   int64_t ld_y, void* y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (int rc = check_weights(weights_host)) return rc;
    const lbfgsb_weights4* w = weights_host;
    if (tokens < 0 || tokens > kMaxRows) return fail(LBFGSB_E_INVALID_ARG, "tokens must be in 0..2^31-1 (got %lld)", (long long)tokens);
    if (!is_logit_type(x_type) || (y_type != x_type && y_type != LBFGSB_F32))
        return fail(LBFGSB_E_INVALID_ARG, "x must be of a logits type and y of the same or F32 (got %d, %d)", x_type, y_type);
    if (tokens == 0) return LBFGSB_OK;
    if (tokens > 1 && (ld_x < w->cols || ld_x > kMaxLd || ld_y < w->rows || ld_y > kMaxLd))
        return fail(LBFGSB_E_INVALID_ARG, "ld_x must be in cols..2^31 and ld_y in rows..2^31 (got %lld, %lld)", (long long)ld_x, (long long)ld_y);
    if (!packed || misaligned(packed, 16)) return fail(LBFGSB_E_INVALID_ARG, "packed is NULL or not aligned to 16 bytes");
    if (!x || !y || misaligned(x, size_of(x_type)) || misaligned(y, size_of(y_type)))
        return fail(LBFGSB_E_INVALID_ARG, "x or y is NULL or not aligned to its elements");
    const Packed4 p = packed_of(w);
    const size_t nx = ((tokens - 1) * ld_x + w->cols) * size_of(x_type), ny = ((tokens - 1) * ld_y + w->rows) * size_of(y_type);
    if (int rc = check_space(matvec4_bytes(p, tokens, x_type), workspace, workspace_bytes)) return rc;
    if (overlap(x, nx, y, ny) || overlap(packed, p.bytes(), y, ny)) return fail(LBFGSB_E_INVALID_ARG, "y overlaps x or packed");
    HIP_TRY(launch_matvec4({p, packed, tokens, ld_x, ld_y, x, y, y_type, workspace}, x_type, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

size_t lbfgsb_draw_workspace_bytes(const lbfgsb_logits* logits_host) {
    if (check_shape(logits_host) || logits_host->vocab > kMaxDrawVocab) return 0;
    return draw_space(logits_host->rows, logits_host->vocab, (int)size_of(logits_host->dtype));
}

int lbfgsb_draw_tokens(const lbfgsb_logits* logits_host, const float* uniform, int64_t* tokens, float* logp, void* workspace, size_t workspace_bytes,
                       void* hip_stream) {
    const lbfgsb_logits* l = logits_host;
    if (int rc = check_logits(l, -1)) return rc;
    if (l->vocab > kMaxDrawVocab) return fail(LBFGSB_E_INVALID_ARG, "tokens are drawn from a vocabulary of at most 2^21 (got %lld)", (long long)l->vocab);
    const int size = (int)size_of(l->dtype);
    if (int rc = check_space(draw_space(l->rows, l->vocab, size), workspace, workspace_bytes)) return rc;
    if (l->rows == 0) return LBFGSB_OK;
    if (!uniform || !tokens || !logp) return fail(LBFGSB_E_INVALID_ARG, "uniform, tokens and logp must not be NULL");
    const double s = 1.0 / l->temperature;
    HIP_TRY(launch_draw({l->z, l->rows, l->ld, (int)l->vocab, s, factor_of(s), uniform, tokens, logp}, l->dtype, workspace, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

size_t lbfgsb_verify_workspace_bytes(const lbfgsb_drafts* drafts_host) { return check_drafts(drafts_host) ? 0 : space_of(drafts_host).whole; }

int lbfgsb_verify_draft(const lbfgsb_drafts* drafts_host, int64_t* tokens, int64_t* count, float* logp, void* workspace, size_t workspace_bytes,
                        void* hip_stream) {
    const lbfgsb_drafts* d = drafts_host;
    if (int rc = check_drafts(d)) return rc;
    if (int rc = check_temperature(d->temperature)) return rc;
    if (d->draft_z)
        if (int rc = check_temperature(d->draft_temperature)) return rc;
    if (int rc = check_strides(d, d->ld, d->ld_request, d->drafts + 1, "logits")) return rc;
    if (d->draft_z)
        if (int rc = check_strides(d, d->draft_ld, d->draft_ld_request, d->drafts, "draft logits")) return rc;
    if (!d->draft_z && d->draft_logp) return fail(LBFGSB_E_INVALID_ARG, "draft_logp goes with draft_z");
    if (int rc = check_space(space_of(d).whole, workspace, workspace_bytes)) return rc;
    if (d->requests == 0) return LBFGSB_OK;
    const size_t b = size_of(d->dtype);
    if (!d->z || misaligned(d->z, b) || misaligned(d->draft_z, b)) return fail(LBFGSB_E_INVALID_ARG, "z is NULL, or z or draft_z not aligned to its elements");
    if (!tokens || !count || !logp || !d->last_uniform || (d->drafts > 0 && (!d->drafted || !d->uniform)))
        return fail(LBFGSB_E_INVALID_ARG, "tokens, count, logp, drafted, uniform and last_uniform must not be NULL");
    VerifyArgs a;
    a.target = {d->z, d->ld, d->ld_request, (int)d->drafts + 1};
    a.draft = {d->drafts > 0 ? d->draft_z : nullptr, d->draft_ld, d->draft_ld_request, (int)d->drafts};
    a.requests = d->requests;
    a.drafts = (int)d->drafts;
    a.vocab = (int)d->vocab;
    a.s = 1.0 / d->temperature;
    a.draft_s = a.draft.z ? 1.0 / d->draft_temperature : 1.0;
    a.c = factor_of(a.s);
    a.draft_c = factor_of(a.draft_s);
    a.draft_logp = d->draft_logp;
    a.drafted = d->drafted;
    a.lengths = d->lengths;
    a.uniform = d->uniform;
    a.last_uniform = d->last_uniform;
    a.tokens = tokens;
    a.count = count;
    a.logp = logp;
    HIP_TRY(launch_verify(a, d->dtype, workspace, (hipStream_t)hip_stream));
    return LBFGSB_OK;
}

}  // extern "C"
