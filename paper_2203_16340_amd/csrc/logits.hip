// The losses on rows of logits: launches by element type, and the totals.
#include "logits.h"

namespace lb {

namespace {

// One workgroup, so that the order of the sum is fixed: 4.7 us for 8192 rows, 1.4 for a few.
constexpr int kTotalBlock = 1024;

__global__ __launch_bounds__(kTotalBlock) void k_weighted_total(const float* row_loss, const float* weight, int64_t n, double scale,
                                                                float* loss, Ascending of) {
    __shared__ double lds[kTotalBlock / 64];
    double sum = 0.0;
    for (int64_t i0 = threadIdx.x; i0 < n; i0 += 4 * kTotalBlock) {
        float v[4], w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t i = i0 + k * kTotalBlock;
            v[k] = i < n ? row_loss[i] : 0.0f;
            w[k] = i < n && weight ? weight[i] : 1.0f;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (w[k] != 0.0f) sum += (double)w[k] * (double)v[k];   // (what does not count may be infinite)
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (of.grad) {
        int descend = 0;
        for (int64_t i = threadIdx.x; i < of.answers; i += kTotalBlock)
            descend |= into(of.offsets[i + 1], of.tokens) < into(of.offsets[i], of.tokens);
        // (answers that share tokens: which of them wrote a token's gradient last would be chance)
        if (__syncthreads_or(descend))
            for (int64_t t = threadIdx.x; t < of.tokens; t += kTotalBlock) of.grad[t] = NAN;
    }
    if (threadIdx.x == 0) {
        double total = 0.0;
        for (int w = 0; w < kTotalBlock / 64; ++w) total += lds[w];
        *loss = (float)(total * scale);
    }
}

// f(value of the element type)
template <typename F>
hipError_t by_type(int dtype, F f) {
    return dtype == LBFGSB_F32 ? f(float{}) : (dtype == LBFGSB_BF16 ? f(__bf16{}) : f(_Float16{}));
}

}  // namespace

int row_splits(int64_t rows, int64_t vocab, int size, bool grad) {
    // Calls in a row on R rows of V bf16 logits, us, whole / in pieces: policy loss with gradient 1 x 16384 7.4 / 6.2, 64 x 16384
    // 8.4 / 7.1, 1 x 32768 9.0 / 8.0, 64 x 32768 9.9 / 8.3, 1 x 131072 19.3 / 7.4, 64 x 131072 20.0 / 10.8; but 64 x 8192 6.5 / 6.9.  Log-probabilities
    // (one launch against two, and less to do in them) 8 x 32768 4.7 / 6.4, 1 x 131072 9.7 / 6.9, 64 x 131072 22 / 8.
    const int64_t chunks = vocab * size / 16;
    if (rows > kSplitRows || chunks < (grad ? 4096 : 8192)) return 1;
    // about two workgroups a compute unit, with two chunks a thread or more
    const int64_t most = chunks / 1024, want = 512 / rows, splits = want < most ? want : most;
    return (int)(splits < kSplits ? splits : kSplits);
}

hipError_t launch_weighted_total(const float* row_loss, const float* weight, int64_t n, double scale, float* loss, hipStream_t st,
                                 const Ascending& of) {
    hipLaunchKernelGGL(k_weighted_total, dim3(1), dim3(kTotalBlock), 0, st, row_loss, weight, n, scale, loss, of);
    return hipGetLastError();
}

hipError_t launch_token_logprob(const LogitsArgs& l, int dtype, const TokenArgs& a, SplitRow* ws, hipStream_t st) {
    if (l.rows == 0) return hipSuccess;
    return by_type(dtype, [&](auto e) { return token_logprob_rows<decltype(e)>(l, a, ws, st); });
}

hipError_t launch_token_logprob_grad(const LogitsArgs& l, int dtype, const TokenGradArgs& a, hipStream_t st) {
    if (l.rows == 0) return hipSuccess;
    return by_type(dtype, [&](auto e) { return token_grad_rows<decltype(e)>(l, a, st); });
}

hipError_t launch_policy(const LogitsArgs& l, int dtype, const PolicyArgs& a, float* loss, SplitRow* ws, hipStream_t st) {
    if (l.rows == 0) return launch_weighted_total(nullptr, nullptr, 0, a.scale, loss, st);
    return by_type(dtype, [&](auto e) { return policy_rows<decltype(e)>(l, a, loss, ws, st); });
}

hipError_t launch_distill(const LogitsArgs& l, int dtype, const DistillArgs& a, float* loss, SplitRow* ws, hipStream_t st) {
    if (l.rows == 0) return launch_weighted_total(nullptr, nullptr, 0, a.scale, loss, st);
    return by_type(dtype, [&](auto e) { return distill_rows<decltype(e)>(l, a, loss, ws, st); });
}

}  // namespace lb
