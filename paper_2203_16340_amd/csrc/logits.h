// Rows of logits: loading, the running maximum and sums of a softmax, and what the losses on a vocabulary
// (token log-probabilities, distillation, policy, preference) share.
#pragma once

#include "common.h"

namespace lb {

constexpr int kMaxTop = 1024;                  // teacher entries of a row, at most
constexpr int64_t kMaxDistillVocab = 1 << 19;  // one bit for each entry of the vocabulary is kept in LDS

// Statistics of a softmax over the entries seen so far, with a_j = (z_j - m) c: m = max z_j, s = sum 2^a_j, t = sum a_j 2^a_j (for
// the entropy).  The difference is taken before the scale, so that a maximum near the type's largest or lowest value overflows
// nothing.
struct Stat {
    float m, s, t;
};

// What a row's entries of the teacher come to.
struct Teacher {
    double cross;       // sum_k q_k (log q_k - s (z_k - z_top))
    double sum;         // sum_k q_k
    float z_top;        // the largest of the student's logits there (0 where all are -infinity)
    Stat top;           // the student's statistics over the entries, each once
    int entries;        // how many there are, each once
    int lost;           // one of them lies past the vocabulary
};

// A few long rows are split: workgroups of a first launch take the statistics of pieces, those of a second join them and write the
// gradient.  What the first leaves for the second, a row each, in the caller's workspace.
constexpr int kSplitRows = 64;      // rows, at most (a wave looks after their total)
constexpr int kSplits = 64;         // pieces of a row, at most (a wave joins them)
struct SplitRow {
    Stat part[kSplits];
    Teacher teacher;
    float zy;                       // the label's logit
    int at[kMaxTop];                // the teacher's entries, as in TopLds
    float q[kMaxTop], z[kMaxTop];
};

// s log2(e), exponentials being powers of two here.  Rounded to 32 bits its error, of one sign and up to 2^-24 of it, puts ln S off by that times
// the mean exponent in every row alike, 6e-8 at temperature 1, which adds up over an answer's tokens.  Entries take c alone, as a difference
// to the largest of their thread; what leads from there to the largest of the row takes both parts, which leaves 1e-8.  (Both parts at
// every entry cost log-probabilities of 8192 x 131072 bf16 with the entropy 322 / 340 us, without 305 / 310.)
struct Factor {
    float c, low;           // the nearest, and what is left
    __device__ __forceinline__ float operator()(float d) const { return fmaf(d, c, d * low); }
};
struct LogitsArgs {
    const void* z;
    void* dz;               // null: no gradient
    int64_t rows, ld, ld_dz;
    int vocab;
    double s;               // 1 / temperature
    Factor c;               // of exponents
};

struct TokenArgs {
    const int64_t* labels;
    float *logp, *lse, *lse_rest, *entropy, *top, *sum;    // all but the first two null: not wanted
};
struct TokenGradArgs {
    const int64_t* labels;
    const float *top, *sum;                    // Stat::m and s; null: from what follows
    const float *lse, *lse_rest;               // lse_rest null: 0
    const float *entropy, *d_logp, *d_entropy; // d_entropy null: no gradient through the entropy
    double temperature;
};
struct DistillArgs {
    const void *index, *logit;
    const float *lse, *weight;                 // either may be null
    float* row_loss;
    int64_t ld;
    int top, index_type, logit_type;
    double scale;
};
struct PolicyArgs {
    const int64_t* labels;
    const float *old_logp, *advantage, *ref_logp, *weight;
    float *row_loss, *logp, *entropy;
    float low, high, kl_coef, entropy_coef;
    int kl_kind;
    double scale;
};
struct PreferenceArgs {
    int64_t tokens, pairs;
    const float *logp, *ref_logp, *weight;
    const int64_t* offsets;
    const uint8_t* mask;
    float *pair_loss, *rewards, *grad;
    double beta, smoothing, margin, scale;
    int kind, normalised;
};

hipError_t launch_token_logprob(const LogitsArgs& l, int dtype, const TokenArgs& a, SplitRow* ws, hipStream_t st);
hipError_t launch_token_logprob_grad(const LogitsArgs& l, int dtype, const TokenGradArgs& a, hipStream_t st);
hipError_t launch_distill(const LogitsArgs& l, int dtype, const DistillArgs& a, float* loss, SplitRow* ws, hipStream_t st);
hipError_t launch_policy(const LogitsArgs& l, int dtype, const PolicyArgs& a, float* loss, SplitRow* ws, hipStream_t st);
hipError_t launch_preference(const PreferenceArgs& a, float* loss, hipStream_t st);
// the same for one element type, rows > 0 (logits_rows.h)
template <typename T>
hipError_t token_logprob_rows(const LogitsArgs& l, const TokenArgs& a, SplitRow* ws, hipStream_t st);
template <typename T>
hipError_t token_grad_rows(const LogitsArgs& l, const TokenGradArgs& a, hipStream_t st);
template <typename T>
hipError_t policy_rows(const LogitsArgs& l, const PolicyArgs& a, float* loss, SplitRow* ws, hipStream_t st);
template <typename T>
hipError_t distill_rows(const LogitsArgs& l, const DistillArgs& a, float* loss, SplitRow* ws, hipStream_t st);
// Offsets of answers that are to ascend, 0 .. tokens, and the gradient that is no number where they do not.
struct Ascending {
    const int64_t* offsets;
    int64_t answers, tokens;
    float* grad;            // null: nothing to do
};
__host__ __device__ inline int64_t into(int64_t v, int64_t tokens) { return v < 0 ? 0 : (v > tokens ? tokens : v); }
// loss = scale * sum_n weight_n row_loss_n
hipError_t launch_weighted_total(const float* row_loss, const float* weight, int64_t n, double scale, float* loss, hipStream_t st,
                                 const Ascending& of = {});
// Pieces that each of a call's rows is split into; 1: none is.
int row_splits(int64_t rows, int64_t vocab, int size, bool grad);   // size: bytes of a logit; grad: a gradient is wanted

// ---- a chunk is 16 bytes of a row ------------------------------------------------------------------------------------
template <typename T>
struct Chunk {
    static constexpr int E = 16 / (int)sizeof(T);
    typedef T vec __attribute__((ext_vector_type(E)));
    typedef vec any __attribute__((aligned(sizeof(T))));           // a row may start on any element
    typedef float wide __attribute__((ext_vector_type(E)));
};

// ---- statistics of a softmax -----------------------------------------------------------------------------------------
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// (how far below the maximum, in powers of two: no further than counts, so that 0 times it is 0; -infinity - -infinity, which is
// no number, ends here as well.  The factor's second part counts only where the first has told that the distance does: times one to the type's
// lowest value it may be past the end, to the other side)
__device__ __forceinline__ float below(float m, float top, Factor c) {
    const float d = m - top;
    return d * c.c > -1000.0f ? fmaxf(c(d), -1000.0f) : -1000.0f;
}
__device__ __forceinline__ Stat rescaled(Stat a, float top, Factor c) {
    const float d = below(a.m, top, c), f = exp2_hw(d);
    return {top, a.s * f, (a.t + d * a.s) * f};
}
__device__ __forceinline__ Stat merged(Stat a, Stat b, Factor c) {
    const float top = fmaxf(a.m, b.m);
    const Stat x = rescaled(a, top, c), y = rescaled(b, top, c);
    return {top, x.s + y.s, x.t + y.t};
}
// what an entry's difference is taken from: 0 where nothing but -infinity was seen, so that such entries stay at 2^-infinity = 0
__device__ __forceinline__ float anchor(float m) { return m == -INFINITY ? 0.0f : m; }

template <int CTRL>
__device__ __forceinline__ float dpp_move_f(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_bcast_f(float v, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); }
__device__ __forceinline__ float wave_max_f(float v) {
    v = fmaxf(v, dpp_move_f<kDppXor1>(v));
    v = fmaxf(v, dpp_move_f<kDppXor2>(v));
    v = fmaxf(v, dpp_move_f<kDppHalfMirror>(v));
    v = fmaxf(v, dpp_move_f<kDppMirror>(v));
    return fmaxf(fmaxf(lane_bcast_f(v, 0), lane_bcast_f(v, 16)), fmaxf(lane_bcast_f(v, 32), lane_bcast_f(v, 48)));
}
__device__ __forceinline__ float wave_sum_f(float v) {
    v += dpp_move_f<kDppXor1>(v);
    v += dpp_move_f<kDppXor2>(v);
    v += dpp_move_f<kDppHalfMirror>(v);
    v += dpp_move_f<kDppMirror>(v);
    return ((lane_bcast_f(v, 0) + lane_bcast_f(v, 16)) + lane_bcast_f(v, 32)) + lane_bcast_f(v, 48);
}
template <bool ENT>
__device__ __forceinline__ Stat wave_stat(Stat a, Factor c) {
    const float top = wave_max_f(a.m);
    a = rescaled(a, top, c);
    return {top, wave_sum_f(a.s), ENT ? wave_sum_f(a.t) : 0.0f};
}
// Joins the statistics of a workgroup's threads; every thread gets the result, in a fixed order.  One barrier; `lds` must not be
// in use by an earlier call any more.
template <bool ENT, int NW>
__device__ __forceinline__ Stat block_stat(Stat a, Factor c, Stat* lds) {
    a = wave_stat<ENT>(a, c);
    if constexpr (NW == 1) {
        __syncthreads();            // (callers count on the barrier)
        return a;
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    float top = lds[0].m;
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, lds[w].m);
    Stat r{top, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
        const Stat x = rescaled(lds[w], top, c);
        r.s += x.s;
        if (ENT) r.t += x.t;
    }
    return r;
}

// A thread's statistics while it goes through its entries.  ref: what an entry's difference is taken from (anchor(a.m)).
struct Running {
    Stat a{-INFINITY, 0.0f, 0.0f};
    float ref = 0.0f;
    template <bool ENT, int N>
    __device__ __forceinline__ void take(const float (&z)[N], Factor c) {
        float top = z[0];
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, z[i]);
        if (top > a.m) {
            const float d = fmaxf((a.m - top) * c.c, -1000.0f), f = exp2_hw(d);      // (c alone, as at its entries)
            a = {top, a.s * f, (a.t + d * a.s) * f};
            ref = top;
        }
        float s[N], t = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = (z[i] - ref) * c.c;
            s[i] = exp2_hw(d);
            if (ENT) t = fmaf(s[i], fmaxf(d, -1000.0f), t);
        }
#pragma unroll
        for (int w = 1; w < N; w *= 2)
#pragma unroll
            for (int i = 0; i + w < N; i += 2 * w) s[i] += s[i + w];
        a.s += s[0];
        if (ENT) a.t += t;
    }
};

// What follows from a row's statistics, in 64 bits.
struct RowLog {
    double log_s, lse, entropy;
};
__device__ __forceinline__ RowLog row_log(Stat a, double s) {
    if (a.s == 0.0f) return {-INFINITY, -INFINITY, 0.0};
    const double ls = log_d((double)a.s);
    return {ls, (double)a.m * s + ls, ls - 0.69314718055994530942 * ((double)a.t / (double)a.s)};
}

}  // namespace lb
