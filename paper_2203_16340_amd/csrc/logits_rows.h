// The kernels of the losses on rows of logits: token log-probabilities and their way back, the clipped policy loss, distillation
// from a teacher's top logits.  Included once for each element type.
//
// With a_j = (z_j - m) c, m the row's maximum, S = sum_j 2^a_j, T = sum_j a_j 2^a_j (Stat in logits.h):
//     lse = m s + ln S,   p_j = 2^a_j / S,   H = ln S - ln 2 T / S,
// and every gradient here is, away from a few marked entries, 2^a_j (A + B a_j) with numbers A, B of the row.
#pragma once

#include <type_traits>

#include "logits.h"

namespace lb {

namespace {

constexpr int64_t kRowBlocksMax = 1 << 20;   // workgroups of a launch, at most: longer batches take several

template <typename T>
__device__ __forceinline__ typename Chunk<T>::wide widened(typename Chunk<T>::vec v) {
    return __builtin_convertvector(v, typename Chunk<T>::wide);
}

// 2^a (A + B a) at a = (z - ref) c
template <bool ENT>
__device__ __forceinline__ float slope_at(float z, float ref, float c, float A, float B) {
    const float d = (z - ref) * c, x = exp2_hw(d);
    return ENT ? x * fmaf(B, fmaxf(d, -1000.0f), A) : x * A;
}

// How a row is cut into chunks: `head` single elements, `whole` chunks that start on 16-byte boundaries of the logits, `tail` single
// elements.  (Loads and stores may start on any element, and stores do where a gradient's rows lie differently; but at
// 50021 16-bit logits a row, which has chunks everywhere if they start with the row, they cost a quarter of the time.  The
// order of the sums depends on where the logits are, not on where the gradient goes.)
template <typename T>
struct Cut {
    static constexpr int E = Chunk<T>::E;
    int head, whole, tail;
    __device__ __forceinline__ Cut(const T* at, int vocab) {
        head = (int)((16u - (unsigned)((uintptr_t)at & 15u)) & 15u) / (int)sizeof(T);
        head = head < vocab ? head : vocab;
        whole = (vocab - head) / E;
        tail = vocab - head - whole * E;
    }
    // the single element of thread t < 2 E, or -1
    __device__ __forceinline__ int single(int t) const {
        return t < E ? (t < head ? t : -1) : (t - E < tail ? head + whole * E + t - E : -1);
    }
    __device__ __forceinline__ int first(int i) const { return head + i * E; }
    // for masks of one bit an entry, so that a chunk's bits stand together: entry j has bit j + shift()
    __device__ __forceinline__ int shift() const { return (E - head) & (E - 1); }
};

// A workgroup's hold on one row.  CH chunks a thread stay in registers between the statistics and the gradient; what a longer row has
// before them is read a second time.  (CH = 0: no gradient, two loads in flight.)
// Loads that are the last of their row go past the caches, unless a workgroup of 1024 makes them: us without / with, token
// log-probabilities of 16400 x 131072 bf16 702 / 665, distillation 4096 x 65536 bf16 208 / 199, but policy 8192 x 131072 bf16 839 / 863.
template <typename T, int BLOCK, int CH>
struct Row {
    static constexpr int E = Chunk<T>::E;
    static constexpr int kSlots = CH > 0 ? CH : 2;
    static constexpr bool NT_LOADS = BLOCK <= 512;
    typedef typename Chunk<T>::vec vec;
    typedef typename Chunk<T>::any any;

    vec slot[kSlots];
    float alone;                         // the single element of this thread, if any
    const char* base;                    // the first chunk
    Cut<T> cut;
    int again;                           // chunks that are read twice

    __device__ __forceinline__ Row(const T* row, int vocab) : cut(row, vocab) {
        base = (const char*)(row + cut.head);
        again = CH > 0 ? (cut.whole > BLOCK * CH ? cut.whole - BLOCK * CH : 0) : cut.whole;
        alone = 0.0f;
        const int j = cut.single((int)threadIdx.x);
        if (j >= 0) alone = (float)row[j];
        start();
    }
    __device__ __forceinline__ vec chunk(int i) const {
        const any* p = (const any*)(base + (size_t)(unsigned)i * 16);
        if constexpr (NT_LOADS) return __builtin_nontemporal_load(p);
        else return *p;
    }
    // Chunk of slot k in the round that begins at chunk `from`, of those before `end`; past the end it is the last one again, which
    // is not looked at.  (No branch: with one around each load the compiler moves it to where its value is used.)
    __device__ __forceinline__ void fetch(int k, int from, int end) {
        const int i = from + k * BLOCK + (int)threadIdx.x;
        slot[k] = chunk(i < end ? i : end - 1);
    }
    __device__ __forceinline__ void start() {
        const int end = again > 0 ? again : cut.whole;
        if (end > 0) {
#pragma unroll
            for (int k = 0; k < kSlots; ++k) fetch(k, 0, end);
        }
    }
    // (the same bits, but to the compiler a new value: else it keeps the 32-bit values of a 16-bit row as well, twice the registers)
    static __device__ __forceinline__ vec opaque(vec v) {
        asm volatile("" : "+v"(v));
        return v;
    }

    // Statistics of the row; ends with the last CH chunks a thread in the slots.  skip (where SKIP): a bit for each entry that stays out
    // (Cut::shift).
    template <bool ENT, bool SKIP>
    __device__ __forceinline__ Stat stat(float c, const unsigned char* skip) {
        Stat a{-INFINITY, 0.0f, 0.0f};
        auto one = [&](vec raw, int i) {
            const auto v = widened<T>(raw);
            float z[E];
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = v[e];
            if constexpr (SKIP) {
                const int at = cut.first(i) + cut.shift();
                const unsigned bits = E == 8 ? skip[at >> 3] : (skip[at >> 3] >> (at & 4)) & 15u;
                if (bits) {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (bits >> e & 1) z[e] = -INFINITY;
                }
            }
            take<ENT>(a, z, c);
        };
        const int j = cut.single((int)threadIdx.x);
        for (int from = 0; from < again; from += BLOCK * kSlots) {
            const int next = from + BLOCK * kSlots;
#pragma unroll
            for (int k = 0; k < kSlots; ++k) {
                const int i = from + k * BLOCK + (int)threadIdx.x;
                if (i < again) one(slot[k], i);
                if (next < again) fetch(k, next, again);
                else if (CH > 0) fetch(k, again, cut.whole);
            }
        }
        if constexpr (CH > 0) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int i = again + k * BLOCK + (int)threadIdx.x;
                if (i < cut.whole) one(slot[k], i);
            }
        }
        if (j >= 0) {
            const float z[1] = {SKIP && (skip[(j + cut.shift()) >> 3] >> ((j + cut.shift()) & 7) & 1) ? -INFINITY : alone};
            take<ENT>(a, z, c);
        }
        return a;
    }

    // dz_j = 2^((z_j - m) c) (A + B (z_j - m) c), and `mark` more at j = y
    template <bool ENT>
    __device__ __forceinline__ void write(T* out, float m, float c, float A, float B, int y, float mark) {
        const float ref = anchor(m);
        char* to = (char*)(out + cut.head);
        auto one = [&](vec raw, int i) {
            const auto v = widened<T>(raw);
            typename Chunk<T>::wide g;
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = slope_at<ENT>(v[e], ref, c, A, B);
            const int at = y - cut.first(i);
            if (at >= 0 && at < E) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (e == at) g[e] += mark;
            }
            __builtin_nontemporal_store(__builtin_convertvector(g, vec), (any*)(to + (size_t)(unsigned)i * 16));
        };
        const int j = cut.single((int)threadIdx.x);
        if (j >= 0) out[j] = (T)(slope_at<ENT>(alone, ref, c, A, B) + (j == y ? mark : 0.0f));
        static_assert(CH > 0);
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int i = again + k * BLOCK + (int)threadIdx.x;
            if (i < cut.whole) one(opaque(slot[k]), i);
            if (again > 0) fetch(k, 0, again);
        }
        for (int from = 0; from < again; from += BLOCK * kSlots) {
            const int next = from + BLOCK * kSlots;
#pragma unroll
            for (int k = 0; k < kSlots; ++k) {
                const int i = from + k * BLOCK + (int)threadIdx.x;
                if (i < again) one(slot[k], i);
                if (next < again) fetch(k, next, again);
            }
        }
    }

    static __device__ __forceinline__ void fill(T* out, int vocab, float value) {
        const Cut<T> cut(out, vocab);
        vec v;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (T)value;
        for (int i = threadIdx.x; i < cut.whole; i += BLOCK) *(any*)((char*)(out + cut.head) + (size_t)(unsigned)i * 16) = v;
        const int j = cut.single((int)threadIdx.x);
        if (j >= 0) out[j] = (T)value;
    }
};

// ---- token log-probabilities -------------------------------------------------------------------------------------------

template <typename T, bool ENT, int BLOCK>
__global__ __launch_bounds__(BLOCK) void k_token_logprob(LogitsArgs l, TokenArgs a, int64_t first) {
    __shared__ Stat lds[BLOCK / 64];
    const int64_t r = first + blockIdx.x;
    const T* row = (const T*)l.z + r * l.ld;
    const int64_t y = a.labels[r];
    if (y < 0) {
        if (threadIdx.x == 0) {
            a.logp[r] = 0.0f;
            a.lse[r] = 0.0f;
            if (a.lse_rest) a.lse_rest[r] = 0.0f;
            if (ENT) a.entropy[r] = 0.0f;
        }
        return;
    }
    const float zy = y < l.vocab ? (float)row[y] : NAN;
    Row<T, BLOCK, 0> z(row, l.vocab);
    const Stat st = block_stat<ENT, BLOCK / 64>(z.template stat<ENT, false>(l.c, nullptr), l.c, lds);
    if (threadIdx.x == 0) {
        const RowLog g = row_log(st, l.s);
        a.logp[r] = st.s == 0.0f ? (y < l.vocab ? -INFINITY : NAN) : (float)(((double)zy - (double)st.m) * l.s - g.log_s);
        const float lse = (float)g.lse;
        a.lse[r] = lse;
        if (a.lse_rest) a.lse_rest[r] = fabsf(lse) < INFINITY ? (float)(((double)st.m * l.s - (double)lse) + g.log_s) : 0.0f;
        if (ENT) a.entropy[r] = (float)g.entropy;
    }
}

// The way back needs no sums: log p_j = z_j s - lse.  Workgroups take pieces of kGradChunks chunks a thread.
constexpr int kGradBlock = 512, kGradChunks = 2;

template <typename T, bool ENT>
__global__ __launch_bounds__(kGradBlock) void k_token_grad(LogitsArgs l, TokenGradArgs a, int pieces, int64_t first) {
    constexpr int E = Chunk<T>::E;
    typedef typename Chunk<T>::vec vec;
    typedef typename Chunk<T>::any any;
    const int64_t w = first + blockIdx.x, r = w / pieces;
    const int piece = (int)(w - r * pieces);
    const T* row = (const T*)l.z + r * l.ld;
    T* out = (T*)l.dz + r * l.ld_dz;
    const Cut<T> cut(row, l.vocab);
    const char* from = (const char*)(row + cut.head);
    char* to = (char*)(out + cut.head);
    const int i0 = piece * (kGradBlock * kGradChunks) + (int)threadIdx.x;
    const int j = piece == 0 ? cut.single((int)threadIdx.x) : -1;
    const int64_t y = a.labels[r];
    const float lse = a.lse[r], rest = a.lse_rest ? a.lse_rest[r] : 0.0f, s = (float)l.s;
    // (a row without a distribution, a label of none: no gradient; a label past the vocabulary: no number)
    const bool none = y < 0 || lse == -INFINITY;
    const float g = none ? 0.0f : (y < l.vocab ? a.d_logp[r] : NAN);
    const float h = !ENT || none ? 0.0f : a.d_entropy[r], entropy = !ENT || none ? 0.0f : a.entropy[r];
    if (g == 0.0f && h == 0.0f) {
        vec zero;
#pragma unroll
        for (int e = 0; e < E; ++e) zero[e] = (T)0.0f;
#pragma unroll
        for (int k = 0; k < kGradChunks; ++k)
            if (i0 + k * kGradBlock < cut.whole) *(any*)(to + (size_t)(unsigned)(i0 + k * kGradBlock) * 16) = zero;
        if (j >= 0) out[j] = (T)0.0f;
        return;
    }
    vec slot[kGradChunks];
#pragma unroll
    for (int k = 0; k < kGradChunks; ++k)
        if (i0 + k * kGradBlock < cut.whole) slot[k] = __builtin_nontemporal_load((const any*)(from + (size_t)(unsigned)(i0 + k * kGradBlock) * 16));
    // p_j (-g - h (log p_j + H))
    const float A = -(g + h * entropy) * s, B = -h * s;
    auto at = [&](float z) {
        const float lp = fmaf(z, s, -lse) - rest, x = exp2_hw(lp * 1.44269504088896340736f);
        return ENT ? x * fmaf(B, fmaxf(lp, -1000.0f), A) : x * A;
    };
    if (j >= 0) out[j] = (T)(at((float)row[j]) + (j == y ? g * s : 0.0f));
#pragma unroll
    for (int k = 0; k < kGradChunks; ++k) {
        const int i = i0 + k * kGradBlock;
        if (i >= cut.whole) break;
        const auto v = widened<T>(slot[k]);
        typename Chunk<T>::wide o;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = at(v[e]);
        const int64_t mark = y - cut.first(i);
        if (mark >= 0 && mark < E) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e == mark) o[e] = fmaf(g, s, o[e]);
        }
        __builtin_nontemporal_store(__builtin_convertvector(o, vec), (any*)(to + (size_t)(unsigned)i * 16));
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

template <typename T, bool ENT, int BLOCK, int CH>
__global__ __launch_bounds__(BLOCK) void k_policy(LogitsArgs l, PolicyArgs a, int64_t first) {
    __shared__ Stat lds[BLOCK / 64];
    const int64_t r = first + blockIdx.x;
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
        if (l.dz) Row<T, BLOCK, CH>::fill(out, l.vocab, 0.0f);
        return;
    }
    Row<T, BLOCK, CH> z(row, l.vocab);
    const float zy = y < l.vocab ? (float)row[y] : NAN;
    const Stat st = block_stat<ENT, BLOCK / 64>(z.template stat<ENT, false>(l.c, nullptr), l.c, lds);
    const RowLog g = row_log(st, l.s);
    const bool empty = st.s == 0.0f;
    const float logp = empty ? (y < l.vocab ? -INFINITY : NAN) : (float)(((double)zy - (double)st.m) * l.s - g.log_s);
    const TokenLoss t = policy_token(a, r, logp);
    if (threadIdx.x == 0) {
        a.row_loss[r] = ENT ? fmaf(-a.entropy_coef, (float)g.entropy, t.loss) : t.loss;
        a.logp[r] = logp;
        if (ENT && a.entropy) a.entropy[r] = (float)g.entropy;
    }
    if (!l.dz) return;
    if (empty) {
        Row<T, BLOCK, CH>::fill(out, l.vocab, 0.0f);
        return;
    }
    // dz_j = W (slope (1[j = y] - p_j) + c_H p_j (log p_j + H)),  log p_j = ln 2 a_j - ln S
    const float W = (float)((double)w * a.scale * l.s), over = W / st.s;
    const float A = over * (ENT ? fmaf(a.entropy_coef, (float)(g.entropy - g.log_s), -t.slope) : -t.slope);
    const float B = ENT ? over * a.entropy_coef * 0.693147180559945309417f : 0.0f;
    z.template write<ENT>(out, st.m, l.c, A, B, (int)y, W * t.slope);
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
__host__ __device__ inline size_t distill_lds(int top, int vocab) { return (size_t)top * 16 + (size_t)(vocab + 8 + 127) / 128 * 16; }

// Between an LDS write of one lane and a read by another of the same wave.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// By the first wave.  An index that comes twice keeps its first place only, with the sum of its shares.  The bits of the
// row's indices are set in `seen`, `by` further on; CLEAR: the words they are in are cleared first (else all are zero already).
template <typename T, bool CLEAR>
__device__ __forceinline__ void read_teacher(const LogitsArgs& l, const DistillArgs& a, int64_t r, const T* row, int by, TopLds s,
                                             Teacher* out) {
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
        if (CLEAR && j >= 0) s.seen[((int)j + by) >> 5] = 0;
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
        const int place = s.at[k] + by;
        const unsigned bit = 1u << (place & 31);
        twice |= (atomicOr(&s.seen[place >> 5], bit) & bit) != 0;
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

template <typename T, bool REST, int BLOCK, int CH>
__global__ __launch_bounds__(BLOCK) void k_distill(LogitsArgs l, DistillArgs a, int64_t first) {
    __shared__ Stat lds[BLOCK / 64];
    __shared__ Teacher teacher;
    extern __shared__ __align__(16) unsigned char dyn[];
    TopLds s;
    s.at = (int*)dyn;
    s.q = (float*)(s.at + a.top);
    s.z = s.q + a.top;
    s.scratch = s.z + a.top;
    s.seen = (unsigned*)(s.scratch + a.top);
    const int64_t r = first + blockIdx.x;
    const T* row = (const T*)l.z + r * l.ld;
    T* out = (T*)l.dz + r * l.ld_dz;
    const float w = a.weight ? a.weight[r] : 1.0f;
    if (w == 0.0f) {
        if (threadIdx.x == 0) a.row_loss[r] = 0.0f;
        if (l.dz) Row<T, BLOCK, CH>::fill(out, l.vocab, 0.0f);
        return;
    }
    Row<T, BLOCK, CH> z(row, l.vocab);
    if (REST) {
        for (int i = threadIdx.x; i < (l.vocab + 8 + 127) / 128 * 4; i += BLOCK) s.seen[i] = 0;
        __syncthreads();
    }
    if (threadIdx.x < 64) read_teacher<T, !REST>(l, a, r, row, z.cut.shift(), s, &teacher);
    if (REST) __syncthreads();
    const Stat st =
        block_stat<false, BLOCK / 64>(z.template stat<false, REST>(l.c, (const unsigned char*)s.seen), l.c, lds);
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
    if (!l.dz) return;
    if (empty && !teacher.lost) {
        Row<T, BLOCK, CH>::fill(out, l.vocab, 0.0f);
        return;
    }
    const float W = loss != loss ? NAN : (float)((double)w * a.scale * l.s);
    z.template write<false>(out, st.m, l.c, W * A, 0.0f, -1, 0.0f);
    __syncthreads();                          // (the entries' own values come after the row's)
    for (int k = threadIdx.x; k < a.top; k += BLOCK) {
        const int j = s.at[k];
        if (j >= 0) out[j] = (T)(W * (exp2_hw((s.z[k] - anchor(all.m)) * l.c) / all.s - s.q[k]));
    }
}

// f(first row or piece, workgroups) for each launch
template <typename F>
void by_rows(int64_t rows, F f) {
    for (int64_t r = 0; r < rows; r += kRowBlocksMax) f(r, dim3((unsigned)(rows - r < kRowBlocksMax ? rows - r : kRowBlocksMax)));
}

// f(BLOCK, CH) for rows of `vocab` elements whose gradient is wanted
template <typename T, typename F>
void by_width(int vocab, F f) {
    constexpr int E = Chunk<T>::E;
    const int chunks = vocab / E;
    using std::integral_constant;
    if (chunks <= 64 * 4) f(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (chunks <= 128 * 4) f(integral_constant<int, 128>{}, integral_constant<int, 4>{});
    else if (chunks <= 256 * 4) f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    else if (chunks <= 256 * 8) f(integral_constant<int, 256>{}, integral_constant<int, 8>{});
    else if (chunks <= 512 * 8) f(integral_constant<int, 512>{}, integral_constant<int, 8>{});
    else if (chunks <= 512 * 10) f(integral_constant<int, 512>{}, integral_constant<int, 10>{});
    else if (chunks <= 512 * 13) f(integral_constant<int, 512>{}, integral_constant<int, 13>{});
    else if (chunks <= 512 * 16) f(integral_constant<int, 512>{}, integral_constant<int, 16>{});
    else if (chunks <= 1024 * 13) f(integral_constant<int, 1024>{}, integral_constant<int, 13>{});
    else f(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
}

}  // namespace

template <typename T>
hipError_t token_logprob_rows(const LogitsArgs& l, const TokenArgs& a, float*, hipStream_t st) {
    const int chunks = l.vocab / Chunk<T>::E;
    auto launch = [&](auto block) {
        constexpr int BLOCK = decltype(block)::value;
        const auto kernel = a.entropy ? k_token_logprob<T, true, BLOCK> : k_token_logprob<T, false, BLOCK>;
        by_rows(l.rows, [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(BLOCK), 0, st, l, a, first); });
    };
    if (chunks <= 1024) launch(std::integral_constant<int, 64>{});
    else if (chunks <= 4096) launch(std::integral_constant<int, 256>{});
    else launch(std::integral_constant<int, 512>{});
    return hipGetLastError();
}

template <typename T>
hipError_t token_grad_rows(const LogitsArgs& l, const TokenGradArgs& a, hipStream_t st) {
    const int64_t piece = (int64_t)kGradBlock * kGradChunks * Chunk<T>::E, pieces = (l.vocab + piece - 1) / piece;
    const auto kernel = a.d_entropy ? k_token_grad<T, true> : k_token_grad<T, false>;
    by_rows(l.rows * pieces,
            [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kGradBlock), 0, st, l, a, (int)pieces, first); });
    return hipGetLastError();
}

template <typename T>
hipError_t policy_rows(const LogitsArgs& l, const PolicyArgs& a, float*, hipStream_t st) {
    by_width<T>(l.vocab, [&](auto block, auto ch) {
        constexpr int BLOCK = decltype(block)::value, CH = decltype(ch)::value;
        const auto kernel = a.entropy || a.entropy_coef != 0.0f ? k_policy<T, true, BLOCK, CH> : k_policy<T, false, BLOCK, CH>;
        by_rows(l.rows, [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(BLOCK), 0, st, l, a, first); });
    });
    return hipGetLastError();
}

template <typename T>
hipError_t distill_rows(const LogitsArgs& l, const DistillArgs& a, float*, hipStream_t st) {
    const size_t lds = distill_lds(a.top, l.vocab);
    hipError_t err = hipSuccess;
    by_width<T>(l.vocab, [&](auto block, auto ch) {
        constexpr int BLOCK = decltype(block)::value, CH = decltype(ch)::value;
        const auto kernel = a.lse ? k_distill<T, true, BLOCK, CH> : k_distill<T, false, BLOCK, CH>;
        err = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (err != hipSuccess) return;
        by_rows(l.rows, [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(BLOCK), lds, st, l, a, first); });
    });
    return err != hipSuccess ? err : hipGetLastError();
}

}  // namespace lb
