// What the C entries on logits (losses_api.hip, rollouts_api.hip) check alike.
#pragma once

#include <algorithm>
#include <cmath>
#include <limits>

#include "logits.h"

namespace lb {

#define HIP_TRY(expr)                                                                           \
    do {                                                                                        \
        hipError_t e_ = (expr);                                                                 \
        if (e_ != hipSuccess) return fail(LBFGSB_E_HIP, "%s: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

constexpr int64_t kMaxRows = (1ll << 31) - 1, kMaxVocab = 1ll << 30, kMaxLd = 1ll << 31;

inline bool is_logit_type(int dtype) { return dtype == LBFGSB_F32 || dtype == LBFGSB_BF16 || dtype == LBFGSB_F16; }
inline size_t size_of(int dtype) { return dtype == LBFGSB_F32 ? 4 : 2; }
inline bool misaligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

// (the exponents' factor is held in 32 bits: infinite, it makes a number of no row)
inline int check_temperature(double t) {
    if (!(t > 0.0) || !std::isfinite(t) || !std::isfinite((float)(1.44269504088896340736 / t)))
        return fail(LBFGSB_E_INVALID_ARG, "temperature must be positive, finite and above 4.24e-39 (got %g)", t);
    return LBFGSB_OK;
}
inline int check_shape(const lbfgsb_logits* l) {
    if (!l) return fail(LBFGSB_E_INVALID_ARG, "logits is NULL");
    if (!is_logit_type(l->dtype)) return fail(LBFGSB_E_INVALID_ARG, "logits: unknown dtype %d", l->dtype);
    if (l->rows < 0 || l->rows > kMaxRows) return fail(LBFGSB_E_INVALID_ARG, "rows must be in 0..2^31-1 (got %lld)", (long long)l->rows);
    if (l->vocab < 1 || l->vocab > kMaxVocab) return fail(LBFGSB_E_INVALID_ARG, "vocab must be in 1..2^30 (got %lld)", (long long)l->vocab);
    return LBFGSB_OK;
}

// grad: the call writes one; 1: it has to, 0: if there is one, -1: it does not
inline int check_logits(const lbfgsb_logits* l, int grad) {
    if (int rc = check_shape(l)) return rc;
    if (l->ld < l->vocab || l->ld > kMaxLd) return fail(LBFGSB_E_INVALID_ARG, "ld must be in vocab..2^31 (got %lld)", (long long)l->ld);
    if (int rc = check_temperature(l->temperature)) return rc;
    if (l->rows == 0) return LBFGSB_OK;
    const size_t b = size_of(l->dtype);
    if (!l->z || misaligned(l->z, b)) return fail(LBFGSB_E_INVALID_ARG, "z is NULL or not aligned to its elements");
    if (grad < 0 || (!l->grad && !grad)) return LBFGSB_OK;
    if (!l->grad || misaligned(l->grad, b)) return fail(LBFGSB_E_INVALID_ARG, "grad is NULL or not aligned to its elements");
    if (l->ld_grad < l->vocab || l->ld_grad > kMaxLd) return fail(LBFGSB_E_INVALID_ARG, "ld_grad must be in vocab..2^31 (got %lld)", (long long)l->ld_grad);
    const uintptr_t z = (uintptr_t)l->z, g = (uintptr_t)l->grad;
    const uintptr_t nz = ((l->rows - 1) * l->ld + l->vocab) * b, ng = ((l->rows - 1) * l->ld_grad + l->vocab) * b;
    if (z < g + ng && g < z + nz && !(z == g && (l->ld == l->ld_grad || l->rows == 1)))
        return fail(LBFGSB_E_INVALID_ARG, "grad overlaps z without being z");
    return LBFGSB_OK;
}
inline Factor factor_of(double s) {
    const double c = s * 1.44269504088896340736;
    // (never 0, which times -infinity is no number)
    const float high = std::max((float)c, std::numeric_limits<float>::denorm_min()), low = (float)(c - (double)high);
    return {high, low};
}
inline int check_space(size_t need, const void* ws, size_t bytes) {
    if (need == 0) return LBFGSB_OK;
    if (!ws || misaligned(ws, 256)) return fail(LBFGSB_E_INVALID_ARG, "workspace is NULL or not aligned to 256 bytes");
    if (bytes < need) return fail(LBFGSB_E_INVALID_ARG, "workspace too small: %zu bytes, need %zu", bytes, need);
    return LBFGSB_OK;
}

}  // namespace lb
