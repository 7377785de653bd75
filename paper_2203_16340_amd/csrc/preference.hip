// The loss on pairs of answers, from the log-probabilities of their tokens.  One workgroup takes a pair: sums of both answers in
// 64 bits, the loss of delta, and the gradient of every token, which is one number for each answer.  9 bytes a token are
// read and 4 written, against 2 or 4 bytes for every entry of a vocabulary before and after it: 2 pairs of 96 tokens take 4.5 us, 24 pairs of
// 8192 tokens 4.8, which is the launch, three trips to memory (offsets, tokens, tokens again out of the caches) and the sums between.
#include "logits.h"

namespace lb {

namespace {

constexpr int kPairBlock = 512;

struct Span {
    int64_t begin, end;
};
// the tokens of answer i; offsets outside 0 .. tokens are taken to the nearest inside, and an answer whose end comes before its beginning
// is empty.  (Where offsets descend, answers may share tokens; the closing launch looks after their gradient.)
__device__ __forceinline__ Span answer(const PreferenceArgs& a, int64_t i) {
    const int64_t begin = into(a.offsets[i], a.tokens), end = into(a.offsets[i + 1], a.tokens);
    return {begin, end < begin ? begin : end};
}

struct LogRatio {
    double sum, n;
};
__device__ __forceinline__ LogRatio sum_answer(const PreferenceArgs& a, Span sp) {
    LogRatio r{0.0, 0.0};
    for (int64_t t = sp.begin + threadIdx.x; t < sp.end; t += kPairBlock) {
        if (a.mask && !a.mask[t]) continue;
        r.sum += (double)a.logp[t] - (a.ref_logp ? (double)a.ref_logp[t] : 0.0);
        r.n += 1.0;
    }
    return r;
}

// log(1 + exp(-|d|)) + max(0, -d) = -log sigmoid(d)
__device__ __forceinline__ double minus_log_sigmoid(double d) { return log1p_d(exp(-fabs(d))) + (d < 0.0 ? -d : 0.0); }

__global__ __launch_bounds__(kPairBlock) void k_preference(PreferenceArgs a) {
    __shared__ double lds[4][kPairBlock / 64];
    // what comes before the first answer and after the last belongs to none
    if (a.grad && blockIdx.x == 0) {
        const int64_t first = a.pairs > 0 ? answer(a, 0).begin : 0, last = a.pairs > 0 ? answer(a, 2 * a.pairs - 1).end : 0;
        for (int64_t t = threadIdx.x; t < first; t += kPairBlock) a.grad[t] = 0.0f;
        for (int64_t t = last + threadIdx.x; t < a.tokens; t += kPairBlock) a.grad[t] = 0.0f;
    }
    for (int64_t i = blockIdx.x; i < a.pairs; i += gridDim.x) {
        const Span sp[2] = {answer(a, i), answer(a, a.pairs + i)};
        double v[4];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const LogRatio r = sum_answer(a, sp[k]);
            v[2 * k] = wave_sum(r.sum);
            v[2 * k + 1] = wave_sum(r.n);
        }
        __syncthreads();
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < 4; ++k) lds[k][threadIdx.x >> 6] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = 0.0;
            for (int w = 0; w < kPairBlock / 64; ++w) v[k] += lds[k][w];
        }
        const double n[2] = {a.normalised && v[1] > 0.0 ? v[1] : 1.0, a.normalised && v[3] > 0.0 ? v[3] : 1.0};
        const double reward[2] = {a.beta * v[0] / n[0], a.beta * v[2] / n[1]};
        const double d = reward[0] - reward[1] - a.margin;
        double loss, slope;
        if (a.kind == LBFGSB_PAIR_SIGMOID) {
            const double x = exp(-fabs(d)), away = (d < 0.0 ? 1.0 : x) / (1.0 + x);   // sigmoid(-d)
            loss = minus_log_sigmoid(d) + (a.smoothing != 0.0 ? a.smoothing * d : 0.0);
            slope = a.smoothing - away;
        } else if (a.kind == LBFGSB_PAIR_HINGE) {
            loss = d < 1.0 ? 1.0 - d : (d >= 1.0 ? 0.0 : d);
            slope = d < 1.0 ? -1.0 : (d >= 1.0 ? 0.0 : d);
        } else {
            const double x = (d - 0.5) / a.beta;
            loss = x * x;
            slope = 2.0 * x / a.beta;
        }
        if (threadIdx.x == 0) {
            a.pair_loss[i] = (float)loss;
            a.rewards[i] = (float)reward[0];
            a.rewards[a.pairs + i] = (float)reward[1];
        }
        if (!a.grad) continue;
        const double w = a.weight ? (double)a.weight[i] : 1.0;
        const double g = w == 0.0 ? 0.0 : slope * w * a.scale * a.beta;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float gk = (float)((k ? -g : g) / n[k]);
            for (int64_t t = sp[k].begin + threadIdx.x; t < sp[k].end; t += kPairBlock)
                a.grad[t] = !a.mask || a.mask[t] ? gk : 0.0f;
        }
    }
}

}  // namespace

hipError_t launch_preference(const PreferenceArgs& a, float* loss, hipStream_t st) {
    if (a.pairs > 0 || (a.grad && a.tokens > 0)) {
        hipLaunchKernelGGL(k_preference, dim3((unsigned)(a.pairs < 1 ? 1 : (a.pairs < 65536 ? a.pairs : 65536))), dim3(kPairBlock), 0, st, a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return launch_weighted_total(a.pair_loss, a.weight, a.pairs, a.scale, loss, st, {a.offsets, 2 * a.pairs, a.tokens, a.grad});
}

}  // namespace lb
