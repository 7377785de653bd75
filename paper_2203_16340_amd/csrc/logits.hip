// Losses on rows of logits: token log-probabilities and their way back, distillation from a teacher's top logits, the clipped
// policy loss.  One workgroup takes a row; it reads the row once for the statistics of its softmax and, where a
// gradient is wanted, once more to write it.
//
// With a_j = (z_j - m) c, m the row's maximum, S = sum_j 2^a_j, T = sum_j a_j 2^a_j (Stat in logits.h):
//     lse = m s + ln S,   p_j = 2^a_j / S,   H = ln S - ln 2 T / S,
// and every gradient here is, away from a few marked entries, 2^a_j (A + B a_j) with numbers A, B of the row.
#include "logits.h"

namespace lb {

namespace {

constexpr int kRowBlock = 512;
constexpr int kRowBlocksMax = 1 << 20;   // rows beyond are taken in turn

template <typename T>
__device__ __forceinline__ typename Chunk<T>::wide widened(typename Chunk<T>::vec v) {
    return __builtin_convertvector(v, typename Chunk<T>::wide);
}

// Statistics of this thread's part of a row.  skip (or null): one bit for each entry of the vocabulary, set where it stays out.
template <typename T, bool ENT, bool SKIP>
__device__ __forceinline__ Stat scan_row(const T* row, int vocab, float c, const unsigned char* skip) {
    constexpr int E = Chunk<T>::E;
    Stat a{-INFINITY, 0.0f, 0.0f};
    for (int64_t e = (int64_t)threadIdx.x * E; e < vocab; e += kRowBlock * E) {
        const auto v = widened<T>(load_chunk(row, (int)e, vocab));
        float z[E];
#pragma unroll
        for (int i = 0; i < E; ++i) z[i] = v[i];
        if constexpr (SKIP) {
            const unsigned bits = E == 8 ? skip[e >> 3] : (skip[e >> 3] >> (e & 4)) & 15u;
            if (bits) {
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (bits >> i & 1) z[i] = -INFINITY;
            }
        }
        take<ENT>(a, z, c);
    }
    return a;
}

// dz_j = 2^((z_j - m) c) (A + B (z_j - m) c), and `mark` more at j = y
template <typename T, bool ENT>
__device__ __forceinline__ void write_row(const T* row, T* out, int vocab, float m, float c, float A, float B, int y, float mark) {
    constexpr int E = Chunk<T>::E;
    const float ref = anchor(m);
    for (int64_t e = (int64_t)threadIdx.x * E; e < vocab; e += kRowBlock * E) {
        const auto v = widened<T>(load_chunk(row, (int)e, vocab));
        typename Chunk<T>::wide g;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float d = (v[i] - ref) * c, x = exp2_hw(d);
            g[i] = ENT ? x * fmaf(B, fmaxf(d, -1000.0f), A) : x * A;
        }
        if (y - (int)e >= 0 && y - (int)e < E) {
#pragma unroll
            for (int i = 0; i < E; ++i)
                if ((int)e + i == y) g[i] += mark;
        }
        store_chunk(out, (int)e, vocab, g);
    }
}

template <typename T>
__device__ __forceinline__ void fill_row(T* out, int vocab, float value) {
    constexpr int E = Chunk<T>::E;
    typename Chunk<T>::wide g;
#pragma unroll
    for (int i = 0; i < E; ++i) g[i] = value;
    for (int64_t e = (int64_t)threadIdx.x * E; e < vocab; e += kRowBlock * E) store_chunk(out, (int)e, vocab, g);
}

// ---- token log-probabilities -------------------------------------------------------------------------------------------

template <typename T, bool ENT>
__global__ __launch_bounds__(kRowBlock) void k_token_logprob(LogitsArgs l, TokenArgs a) {
    __shared__ Stat lds[kRowBlock / 64];
    for (int64_t r = blockIdx.x; r < l.rows; r += gridDim.x) {
        const T* row = (const T*)l.z + r * l.ld;
        const int64_t y = a.labels[r];
        if (y < 0) {
            if (threadIdx.x == 0) {
                a.logp[r] = 0.0f;
                a.lse[r] = 0.0f;
                if (a.lse_rest) a.lse_rest[r] = 0.0f;
                if (ENT) a.entropy[r] = 0.0f;
            }
            continue;
        }
        const float zy = y < l.vocab ? (float)row[y] : NAN;
        __syncthreads();
        const Stat st = block_stat<ENT, kRowBlock / 64>(scan_row<T, ENT, false>(row, l.vocab, l.c, nullptr), l.c, lds);
        if (threadIdx.x == 0) {
            const RowLog g = row_log(st, l.s);
            a.logp[r] = st.s == 0.0f ? (y < l.vocab ? -INFINITY : NAN) : (float)(((double)zy - (double)st.m) * l.s - g.log_s);
            const float lse = (float)g.lse;
            a.lse[r] = lse;
            if (a.lse_rest) a.lse_rest[r] = fabsf(lse) < INFINITY ? (float)(((double)st.m * l.s - (double)lse) + g.log_s) : 0.0f;
            if (ENT) a.entropy[r] = (float)g.entropy;
        }
    }
}

// The way back needs no sums: log p_j = z_j s - lse.  Workgroups take pieces of kGradChunks chunks a thread.
constexpr int kGradBlock = 256, kGradChunks = 4;

template <typename T, bool ENT>
__global__ __launch_bounds__(kGradBlock) void k_token_grad(LogitsArgs l, TokenGradArgs a, int pieces) {
    constexpr int E = Chunk<T>::E;
    const int64_t total = l.rows * pieces;
    for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
        const int64_t r = w / pieces;
        const int64_t first = (w - r * pieces) * (kGradBlock * kGradChunks * E) + (int64_t)threadIdx.x * E;
        const T* row = (const T*)l.z + r * l.ld;
        T* out = (T*)l.dz + r * l.ld_dz;
        const int64_t y = a.labels[r];
        const float lse = a.lse[r], rest = a.lse_rest ? a.lse_rest[r] : 0.0f;
        // (a row without a distribution, a label of none: no gradient; a label past the vocabulary: no number)
        float g = y < 0 || lse == -INFINITY ? 0.0f : (y < l.vocab ? a.d_logp[r] : NAN);
        float h = 0.0f, entropy = 0.0f;
        if (ENT && g == g && y >= 0 && lse != -INFINITY) {
            h = a.d_entropy[r];
            entropy = a.entropy[r];
        }
        const float s = (float)l.s;
        if (g == 0.0f && h == 0.0f) {
            typename Chunk<T>::wide zero = (typename Chunk<T>::wide)(0.0f);
#pragma unroll
            for (int k = 0; k < kGradChunks; ++k) {
                const int64_t e = first + (int64_t)k * kGradBlock * E;
                if (e < l.vocab) store_chunk(out, (int)e, l.vocab, zero);
            }
            continue;
        }
        // p_j (-g - h (log p_j + H))
        const float A = -(g + h * entropy) * s, B = -h * s;
#pragma unroll
        for (int k = 0; k < kGradChunks; ++k) {
            const int64_t e = first + (int64_t)k * kGradBlock * E;
            if (e >= l.vocab) break;
            const auto v = widened<T>(load_chunk(row, (int)e, l.vocab));
            typename Chunk<T>::wide o;
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float lp = fmaf(v[i], s, -lse) - rest, x = exp2_hw(lp * 1.44269504088896340736f);
                o[i] = ENT ? x * fmaf(B, fmaxf(lp, -1000.0f), A) : x * A;
            }
            if (y - e >= 0 && y - e < E) {
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (e + i == y) o[i] = fmaf(g, s, o[i]);
            }
            store_chunk(out, (int)e, l.vocab, o);
        }
    }
}

// ---- policy --------------------------------------------------------------------------------------------------------------

// loss of a token and its derivative with respect to logp, without the entropy's term
struct TokenLoss {
    float loss, slope;
};
__device__ __forceinline__ TokenLoss policy_token(const PolicyArgs& a, int64_t r, float logp) {
    const float ratio = expf(logp - a.old_logp[r]), adv = a.advantage[r];
    const float whole = ratio * adv, held = fminf(fmaxf(ratio, a.low), a.high) * adv;
    // (a ratio that is no number stays one: the minimum would drop it)
    TokenLoss t{whole <= held ? -whole : (whole > held ? -held : whole + held), whole > held ? 0.0f : -whole};
    if (a.kl_coef != 0.0f) {
        const float d = logp - a.ref_logp[r];
        float kl, slope;
        if (a.kl_kind == LBFGSB_KL_1) {
            kl = d;
            slope = 1.0f;
        } else if (a.kl_kind == LBFGSB_KL_2) {
            kl = 0.5f * d * d;
            slope = d;
        } else {
            const float x = expm1f(-d);
            kl = x + d;
            slope = -x;
        }
        t.loss = fmaf(a.kl_coef, kl, t.loss);
        t.slope = fmaf(a.kl_coef, slope, t.slope);
    }
    return t;
}

template <typename T, bool ENT>
__global__ __launch_bounds__(kRowBlock) void k_policy(LogitsArgs l, PolicyArgs a) {
    __shared__ Stat lds[kRowBlock / 64];
    for (int64_t r = blockIdx.x; r < l.rows; r += gridDim.x) {
        const T* row = (const T*)l.z + r * l.ld;
        T* out = (T*)l.dz + r * l.ld_dz;
        const int64_t y = a.labels[r];
        const float w = a.weight ? a.weight[r] : 1.0f;
        if (y < 0 || w == 0.0f) {
            if (threadIdx.x == 0) {
                a.row_loss[r] = 0.0f;
                a.logp[r] = 0.0f;
                if (a.entropy) a.entropy[r] = 0.0f;
            }
            if (l.dz) fill_row(out, l.vocab, 0.0f);
            continue;
        }
        const float zy = y < l.vocab ? (float)row[y] : NAN;
        __syncthreads();
        const Stat st = block_stat<ENT, kRowBlock / 64>(scan_row<T, ENT, false>(row, l.vocab, l.c, nullptr), l.c, lds);
        const RowLog g = row_log(st, l.s);
        const bool empty = st.s == 0.0f;
        const float logp = empty ? (y < l.vocab ? -INFINITY : NAN) : (float)(((double)zy - (double)st.m) * l.s - g.log_s);
        const TokenLoss t = policy_token(a, r, logp);
        if (threadIdx.x == 0) {
            a.row_loss[r] = ENT ? fmaf(-a.entropy_coef, (float)g.entropy, t.loss) : t.loss;
            a.logp[r] = logp;
            if (ENT && a.entropy) a.entropy[r] = (float)g.entropy;
        }
        if (!l.dz) continue;
        if (empty) {
            fill_row(out, l.vocab, 0.0f);
            continue;
        }
        // dz_j = W (slope (1[j = y] - p_j) + c_H p_j (log p_j + H)),  log p_j = ln 2 a_j - ln S
        const float W = (float)((double)w * a.scale * l.s), over = W / st.s;
        const float A = over * (ENT ? fmaf(a.entropy_coef, (float)(g.entropy - g.log_s), -t.slope) : -t.slope);
        const float B = ENT ? over * a.entropy_coef * 0.693147180559945309417f : 0.0f;
        write_row<T, ENT>(row, out, l.vocab, st.m, l.c, A, B, (int)y, W * t.slope);
    }
}

// ---- distillation ----------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float teacher_logit(const DistillArgs& a, int64_t at) {
    return a.logit_type == LBFGSB_F32 ? ((const float*)a.logit)[at]
         : a.logit_type == LBFGSB_BF16 ? (float)((const __bf16*)a.logit)[at] : (float)((const _Float16*)a.logit)[at];
}
__device__ __forceinline__ int64_t teacher_index(const DistillArgs& a, int64_t at) {
    return a.index_type == LBFGSB_I32 ? (int64_t)((const int*)a.index)[at] : ((const int64_t*)a.index)[at];
}

// What a row's first wave finds out about the teacher, in LDS.
struct Teacher {
    double cross;       // sum_k q_k (log q_k - s z_k)
    double sum;         // sum_k q_k
    Stat top;           // the student's statistics over the entries, each once
    int entries;        // how many there are, each once
    int lost;           // one of them lies past the vocabulary
};
// LDS of the distillation kernel: a row's entries (index, teacher's share, student's logit, scratch), then one bit for each
// entry of the vocabulary.
struct TopLds {
    int* at;
    float *q, *z, *scratch;
    unsigned* seen;
};
__host__ __device__ inline size_t distill_lds(int top, int vocab) { return (size_t)top * 16 + (size_t)(vocab + 127) / 128 * 16; }

// Between an LDS write of one lane and a read by another of the same wave.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// By the first wave.  An index that comes twice keeps its first place only, with the sum of its shares.  The bits of the
// row's indices are set in `seen`; CLEAR: the words they are in are cleared first (else all are zero already).
template <typename T, bool CLEAR>
__device__ __forceinline__ void read_teacher(const LogitsArgs& l, const DistillArgs& a, int64_t r, const T* row, TopLds s, Teacher* out) {
    const int lane = threadIdx.x & 63, top = a.top;
    float most = -INFINITY;
    bool lost = false;
    for (int k = lane; k < top; k += 64) {
        int64_t j = teacher_index(a, r * a.ld + k);
        float v = teacher_logit(a, r * a.ld + k);
        lost |= j >= l.vocab;
        if (j < 0 || j >= l.vocab || v == -INFINITY) {
            j = -1;
            v = -INFINITY;
        }
        s.at[k] = (int)j;
        s.q[k] = v;
        s.z[k] = j >= 0 ? (float)row[j] : -INFINITY;
        if (CLEAR && j >= 0) s.seen[j >> 5] = 0;
        most = fmaxf(most, v);
    }
    wave_fence();
    most = anchor(wave_max_f(most));
    const bool given = a.lse != nullptr;
    // log q_k = s (a_k - most) - shift
    double shift;
    if (given) {
        shift = (double)a.lse[r] - (double)most * l.s;
    } else {
        double total = 0.0;
        for (int k = lane; k < top; k += 64)
            if (s.at[k] >= 0) total += (double)exp2_hw((s.q[k] - most) * l.c);
        total = wave_sum(total);
        shift = total > 0.0 ? log_d(total) : total;
    }
    double cross = 0.0, sum = 0.0;
    bool twice = false;
    for (int k = lane; k < top; k += 64) {
        if (s.at[k] < 0) continue;
        const double lq = ((double)s.q[k] - (double)most) * l.s - shift;
        const float qk = expf((float)lq);
        s.q[k] = qk;
        sum += (double)qk;
        if (qk != 0.0f) cross += (double)qk * (lq - (double)s.z[k] * l.s);
        const unsigned bit = 1u << (s.at[k] & 31);
        twice |= (atomicOr(&s.seen[s.at[k] >> 5], bit) & bit) != 0;
    }
    wave_fence();
    if (__any(twice)) {
        unsigned again = 0;                       // one bit for each of this lane's entries (kMaxTop / 64 = 16 of them)
        for (int k = lane, n = 0; k < top; k += 64, ++n) {
            float share = 0.0f;
            for (int i = 0; i < top; ++i)
                if (s.at[i] == s.at[k]) {
                    share += s.q[i];
                    if (i < k) again |= 1u << n;
                }
            s.scratch[k] = share;
        }
        wave_fence();
        for (int k = lane, n = 0; k < top; k += 64, ++n) {
            s.q[k] = s.scratch[k];
            if (again >> n & 1) s.at[k] = -1;
        }
    }
    Stat st{-INFINITY, 0.0f, 0.0f};
    int entries = 0;
    for (int k = lane; k < top; k += 64)
        if (s.at[k] >= 0) {
            const float v[1] = {s.z[k]};
            take<false>(st, v, l.c);
            ++entries;
        }
    st = wave_stat<false>(st, l.c);
    cross = wave_sum(cross);
    sum = wave_sum(sum);
    const double count = wave_sum((double)entries);
    const int any_lost = __any(lost);
    if (lane == 0) *out = {cross, sum, st, (int)count, any_lost};
}

template <typename T, bool REST>
__global__ __launch_bounds__(kRowBlock) void k_distill(LogitsArgs l, DistillArgs a) {
    __shared__ Stat lds[kRowBlock / 64];
    __shared__ Teacher teacher;
    extern __shared__ __align__(16) unsigned char dyn[];
    TopLds s;
    s.at = (int*)dyn;
    s.q = (float*)(s.at + a.top);
    s.z = s.q + a.top;
    s.scratch = s.z + a.top;
    s.seen = (unsigned*)(s.scratch + a.top);
    for (int64_t r = blockIdx.x; r < l.rows; r += gridDim.x) {
        const T* row = (const T*)l.z + r * l.ld;
        T* out = (T*)l.dz + r * l.ld_dz;
        const float w = a.weight ? a.weight[r] : 1.0f;
        if (w == 0.0f) {
            if (threadIdx.x == 0) a.row_loss[r] = 0.0f;
            if (l.dz) fill_row(out, l.vocab, 0.0f);
            continue;
        }
        __syncthreads();                          // (the last row's entries are done with)
        if (REST) {
            for (int i = threadIdx.x; i < (l.vocab + 127) / 128 * 4; i += kRowBlock) s.seen[i] = 0;
            __syncthreads();
        }
        if (threadIdx.x < 64) read_teacher<T, !REST>(l, a, r, row, s, &teacher);
        if (REST) __syncthreads();
        const Stat st =
            block_stat<false, kRowBlock / 64>(scan_row<T, false, REST>(row, l.vocab, l.c, (const unsigned char*)s.seen), l.c, lds);
        const Stat all = REST ? merged(st, teacher.top, l.c) : st;
        const RowLog g = row_log(all, l.s);
        const bool empty = all.s == 0.0f;
        double loss = teacher.entries ? teacher.cross + teacher.sum * g.lse : 0.0;
        float A;                                  // away from the entries, dz_j = W A 2^((z_j - st.m) c)
        if (REST) {
            // the rest's shares: r of the teacher, t of the student
            const double rest = teacher.entries < l.vocab ? (teacher.sum < 1.0 ? 1.0 - teacher.sum : 0.0) : 0.0;
            const double log_t = st.s == 0.0f ? -INFINITY : ((double)st.m - (double)all.m) * l.s + log_d((double)st.s) - g.log_s;
            if (rest > 0.0) loss += rest * (log_d(rest) - log_t);
            A = st.s == 0.0f ? 0.0f : (float)(((double)expf((float)log_t) - rest) / (double)st.s);
        } else {
            A = teacher.entries ? 1.0f / st.s : 0.0f;
        }
        if (empty) loss = teacher.entries ? INFINITY : 0.0;
        if (teacher.lost) loss = NAN;
        if (threadIdx.x == 0) a.row_loss[r] = (float)loss;
        if (!l.dz) continue;
        if (empty && !teacher.lost) {
            fill_row(out, l.vocab, 0.0f);
            continue;
        }
        const float W = loss != loss ? NAN : (float)((double)w * a.scale * l.s);
        write_row<T, false>(row, out, l.vocab, st.m, l.c, W * A, 0.0f, -1, 0.0f);
        __syncthreads();                          // (the entries' own values come after the row's)
        for (int k = threadIdx.x; k < a.top; k += kRowBlock) {
            const int j = s.at[k];
            if (j >= 0) out[j] = (T)(W * (exp2_hw((s.z[k] - anchor(all.m)) * l.c) / all.s - s.q[k]));
        }
    }
}

// ---- totals ------------------------------------------------------------------------------------------------------------------

constexpr int kTotalBlock = 1024;

__global__ __launch_bounds__(kTotalBlock) void k_weighted_total(const float* row_loss, const float* weight, int64_t n, double scale,
                                                                float* loss) {
    __shared__ double lds[kTotalBlock / 64];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += kTotalBlock) {
        const float w = weight ? weight[i] : 1.0f;
        if (w != 0.0f) sum += (double)w * (double)row_loss[i];   // (what does not count may be infinite)
    }
    sum = wave_sum(sum);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double total = 0.0;
        for (int w = 0; w < kTotalBlock / 64; ++w) total += lds[w];
        *loss = (float)(total * scale);
    }
}

unsigned row_grid(int64_t rows) { return (unsigned)(rows < kRowBlocksMax ? rows : kRowBlocksMax); }

// f(type) for the element type of the logits
template <typename F>
void by_type(int dtype, F f) {
    if (dtype == LBFGSB_F32) f(float{});
    else if (dtype == LBFGSB_BF16) f(__bf16{});
    else f(_Float16{});
}

}  // namespace

size_t logits_workspace(int64_t, int64_t, int) { return 0; }

hipError_t launch_weighted_total(const float* row_loss, const float* weight, int64_t n, double scale, float* loss, hipStream_t st) {
    hipLaunchKernelGGL(k_weighted_total, dim3(1), dim3(kTotalBlock), 0, st, row_loss, weight, n, scale, loss);
    return hipGetLastError();
}

hipError_t launch_token_logprob(const LogitsArgs& l, int dtype, const TokenArgs& a, float*, hipStream_t st) {
    if (l.rows == 0) return hipSuccess;
    by_type(dtype, [&](auto e) {
        using T = decltype(e);
        if (a.entropy) hipLaunchKernelGGL((k_token_logprob<T, true>), dim3(row_grid(l.rows)), dim3(kRowBlock), 0, st, l, a);
        else hipLaunchKernelGGL((k_token_logprob<T, false>), dim3(row_grid(l.rows)), dim3(kRowBlock), 0, st, l, a);
    });
    return hipGetLastError();
}

hipError_t launch_token_logprob_grad(const LogitsArgs& l, int dtype, const TokenGradArgs& a, hipStream_t st) {
    if (l.rows == 0) return hipSuccess;
    by_type(dtype, [&](auto e) {
        using T = decltype(e);
        const int64_t piece = (int64_t)kGradBlock * kGradChunks * Chunk<T>::E, pieces = (l.vocab + piece - 1) / piece;
        const int64_t total = l.rows * pieces;
        const dim3 grid((unsigned)(total < kRowBlocksMax ? total : kRowBlocksMax));
        if (a.d_entropy) hipLaunchKernelGGL((k_token_grad<T, true>), grid, dim3(kGradBlock), 0, st, l, a, (int)pieces);
        else hipLaunchKernelGGL((k_token_grad<T, false>), grid, dim3(kGradBlock), 0, st, l, a, (int)pieces);
    });
    return hipGetLastError();
}

hipError_t launch_policy(const LogitsArgs& l, int dtype, const PolicyArgs& a, float* loss, float*, hipStream_t st) {
    if (l.rows > 0) {
        by_type(dtype, [&](auto e) {
            using T = decltype(e);
            if (a.entropy || a.entropy_coef != 0.0f)
                hipLaunchKernelGGL((k_policy<T, true>), dim3(row_grid(l.rows)), dim3(kRowBlock), 0, st, l, a);
            else
                hipLaunchKernelGGL((k_policy<T, false>), dim3(row_grid(l.rows)), dim3(kRowBlock), 0, st, l, a);
        });
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return launch_weighted_total(a.row_loss, a.weight, l.rows, a.scale, loss, st);
}

hipError_t launch_distill(const LogitsArgs& l, int dtype, const DistillArgs& a, float* loss, float*, hipStream_t st) {
    if (l.rows > 0) {
        const size_t lds = distill_lds(a.top, l.vocab);
        hipError_t err = hipSuccess;
        by_type(dtype, [&](auto e) {
            using T = decltype(e);
            const auto kernel = a.lse ? k_distill<T, true> : k_distill<T, false>;
            err = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (err == hipSuccess) hipLaunchKernelGGL(kernel, dim3(row_grid(l.rows)), dim3(kRowBlock), lds, st, l, a);
        });
        if (err != hipSuccess) return err;
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    return launch_weighted_total(a.row_loss, a.weight, l.rows, a.scale, loss, st);
}

}  // namespace lb
