// The kernels of the losses on rows of logits: token log-probabilities and their way back, the clipped policy loss, distillation
// from a teacher's top logits.  Included once for each element type.
//
// With a_j = (z_j - m) c, m the row's maximum, S = sum_j 2^a_j, T = sum_j a_j 2^a_j (Stat in logits.h):
//     lse = m s + ln S,   p_j = 2^a_j / S,   H = ln S - ln 2 T / S,
// and every gradient here is, away from a few marked entries, 2^a_j (A + B a_j) with numbers A, B of the row.
//
// All of it is bound by memory: 4 to 10 operations and one or two exponentials an entry against 2 or 4 bytes read (and as many
// written).  So a row is read once where it fits a workgroup's registers, in 16-byte chunks a thread with all loads in flight at
// once, and its sums and maxima are taken while they arrive: a maximum and a sum for each thread, joined over the wave by lane
// permutations and over the workgroup through LDS, behind one barrier.  (The exponentials are no bound: with one multiply-add in
// place of a difference and a product in both passes, the times were the same.)
#pragma once

#include <cfloat>

#include <algorithm>
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
__device__ __forceinline__ float slope_at(float z, float ref, Factor c, float A, float B) {
    const float d = (z - ref) * c.c, x = exp2_hw(d);
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
    // chunks from the boundary of a 128-byte line to the first one: with the waves' loads and stores starting on lines (chunk i - lead by
    // thread i), 8192 x 50000 bf16, whose rows do not, takes 284 us for 311
    __device__ __forceinline__ int lead(const T* at) const { return (int)(((uintptr_t)(at + head) >> 4) & 7u); }
    // the single element of thread t < 2 E, or -1
    __device__ __forceinline__ int single(int t) const {
        return t < E ? (t < head ? t : -1) : (t - E < tail ? head + whole * E + t - E : -1);
    }
    __device__ __forceinline__ int first(int i) const { return head + i * E; }
    // for masks of one bit an entry, so that a chunk's bits stand together: entry j has bit j + shift()
    __device__ __forceinline__ int shift() const { return (E - head) & (E - 1); }
};

// A row, or piece `piece` of `pieces` of it, as a workgroup goes through it: what is the same for all its threads.
template <typename T, int HOLD, bool LONG>       // HOLD: chunks that the workgroup keeps; LONG: there may be more of them
struct Span {
    static constexpr int E = Chunk<T>::E;
    static constexpr bool SURE = HOLD >= 8192;       // LONG is only asked for where there are more: a whole row of HOLD - 8 chunks at least
    const T* row;
    Cut<T> cut;
    int begin, end;                      // its chunks
    int again;                           // up to here they are read twice
    int origin, keep;                    // where thread 0 stands in the first round and in what is kept: on a line, up to 7 before the first
    bool singles;                        // the single elements go with the first piece

    __device__ __forceinline__ Span(const T* r, int vocab, int piece = 0, int pieces = 1) : row(r), cut(r, vocab) {
        const int lead = cut.lead(r), each = ((cut.whole + lead + pieces - 1) / pieces + 7) & ~7;
        begin = pieces == 1 || piece == 0 ? 0 : min(piece * each - lead, cut.whole);
        end = pieces == 1 ? cut.whole : max(min((piece + 1) * each - lead, cut.whole), begin);
        origin = begin == 0 ? -lead : begin;
        if (HOLD == 0) again = end;
        else again = LONG && (SURE || end - origin > HOLD) ? max(((end - (HOLD - 16) + lead + 7) & ~7) - lead, begin) : begin;
        keep = repeats() ? again : origin;
        singles = piece == 0;
    }
    __device__ __forceinline__ const char* base() const { return (const char*)(row + cut.head); }
    __device__ __forceinline__ bool repeats() const { return LONG && (SURE || again > begin); }
    // the first chunks that are read: up to here
    __device__ __forceinline__ int first_end() const { return repeats() ? again : end; }
    __device__ __forceinline__ int single() const { return singles ? cut.single((int)threadIdx.x) : -1; }
    // whether element e is one of this piece's
    __device__ __forceinline__ bool has(int e) const {
        const int i = e - cut.head;
        return i < 0 || i >= cut.whole * E ? singles : i >= begin * E && i < end * E;
    }
};

// A workgroup's hold on a span.  CH chunks a thread stay in registers between the statistics and the gradient; what a longer row has
// before them waits in LDS (HELD) or is read a second time.  (CH = 0: no gradient, SLOTS loads in flight.)
// Loads that are the last of their row go past the caches, unless a workgroup of 1024 makes them: us without / with, token
// log-probabilities of 16400 x 131072 bf16 702 / 665, distillation 4096 x 65536 bf16 208 / 199, but policy 8192 x 131072 bf16 839 / 863.
template <typename T, int BLOCK, int CH, bool LONG = CH == 0, bool HELD = false, bool NT_LOADS = (BLOCK <= 512), int SLOTS = 2>
struct Row {
    static constexpr int E = Chunk<T>::E;
    static constexpr int kSlots = CH > 0 ? CH : SLOTS;
    typedef typename Chunk<T>::vec vec;
    typedef typename Chunk<T>::any any;
    typedef lb::Span<T, BLOCK * CH, LONG> Span;

    vec slot[kSlots];
    float alone;                         // the single element of this thread, if any
    vec* held;                           // HELD: room in LDS for the chunks before `again` (held_bytes)

    // The thread's index, to the compiler a new value each time: else it keeps what it worked out for one loop over the slots until the
    // next, one or two registers, which are a wave in the distillation with 13 chunks (80 / 81).
    static __device__ __forceinline__ int thread() {
        int t = (int)threadIdx.x;
        asm volatile("" : "+v"(t));
        return t;
    }
    static __device__ __forceinline__ vec chunk(const Span& sp, int i) {
        const any* p = (const any*)(sp.base() + (size_t)(unsigned)i * 16);
        if constexpr (NT_LOADS) return __builtin_nontemporal_load(p);
        else return *p;
    }
    // Chunk of slot k in the round that thread 0 begins at `from`, of those from `at` on and before `to`; outside it is the first or last
    // one again, which is not looked at.  (No branch: with one around each load the compiler moves it to where its value is used.)
    __device__ __forceinline__ void fetch(const Span& sp, int k, int from, int at, int to, int t) {
        const int i = from + k * BLOCK + t;
        slot[k] = chunk(sp, min(k == 0 ? max(i, at) : i, to - 1));
    }
    static __device__ __forceinline__ bool in(int k, int i, int at, int to) { return (k > 0 || i >= at) && i < to; }
    __device__ __forceinline__ void open_single(const Span& sp) {
        alone = 0.0f;
        const int j = sp.single();
        if (j >= 0) alone = (float)sp.row[j];
    }
    __device__ __forceinline__ void open(const Span& sp) {
        open_single(sp);
        const int to = sp.first_end(), t = thread();
        if (to > sp.begin) {
#pragma unroll
            for (int k = 0; k < kSlots; ++k) fetch(sp, k, sp.origin, sp.begin, to, t);
        }
    }
    // Straight to what write() expects, where the statistics are known already: the last chunks in the slots.
    __device__ __forceinline__ void open_last(const Span& sp) {
        open_single(sp);
        const int t = thread();
        if (sp.end > sp.again) {
#pragma unroll
            for (int k = 0; k < kSlots; ++k) fetch(sp, k, sp.keep, sp.again, sp.end, t);
        }
    }
    // (the same bits, but to the compiler a new value: else it keeps the 32-bit values of a 16-bit row as well, twice the registers)
    static __device__ __forceinline__ vec opaque(vec v) {
        asm volatile("" : "+v"(v));
        return v;
    }

    // Statistics of an open span; ends with the last CH chunks a thread in the slots.  skip (where SKIP): a bit for each entry that stays
    // out (Cut::shift).
    template <bool ENT, bool SKIP>
    __device__ __forceinline__ Stat stat(const Span& sp, Factor c, const unsigned char* skip) {
        Running a;
        auto skipped = [&](int i) -> unsigned {
            const int at = sp.cut.first(i) + sp.cut.shift();
            return E == 8 ? skip[at >> 3] : (skip[at >> 3] >> (at & 4)) & 15u;
        };
        auto one = [&](vec raw, unsigned bits) {
            const auto v = widened<T>(raw);
            float z[E];
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = v[e];
            if constexpr (SKIP) {
                if (bits) {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (bits >> e & 1) z[e] = -INFINITY;
                }
            }
            a.take<ENT>(z, c);
        };
        const int t = thread();
        const int first = CH > 0 ? sp.again : sp.end;
        if (CH == 0 || sp.repeats()) for (int from = sp.origin; from < first; from += BLOCK * kSlots) {
            const int next = from + BLOCK * kSlots;
#pragma unroll
            for (int k = 0; k < kSlots; ++k) {
                const int i = from + k * BLOCK + t;
                if (in(k, i, sp.begin, first)) {
                    if constexpr (HELD) held[i - sp.origin] = slot[k];
                    one(slot[k], SKIP ? skipped(i) : 0);
                }
                if (next < first) fetch(sp, k, next, sp.begin, first, t);
                else if (CH > 0) fetch(sp, k, sp.keep, sp.again, sp.end, t);
            }
        }
        if constexpr (CH > 0) {
            unsigned bits[CH] = {};                   // (all of them asked for before the first is waited for)
            if constexpr (SKIP) {
#pragma unroll
                for (int k = 0; k < CH; ++k) bits[k] = skipped(max(min(sp.keep + k * BLOCK + t, sp.end - 1), 0));
            }
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int i = sp.keep + k * BLOCK + t;
                if (in(k, i, sp.again, sp.end)) one(slot[k], bits[k]);
            }
        }
        const int j = sp.single();
        if (j >= 0) {
            const float z[1] = {SKIP && (skip[(j + sp.cut.shift()) >> 3] >> ((j + sp.cut.shift()) & 7) & 1) ? -INFINITY : alone};
            a.take<ENT>(z, c);
        }
        return a.a;
    }

    // dz_j = 2^((z_j - m) c) (A + B (z_j - m) c), and `mark` more at j = y (none: -1), where the logit is zy.
    template <bool ENT>
    __device__ __forceinline__ void write(const Span& sp, T* out, float m, Factor c, float A, float B, int y, float zy, float mark) {
        static_assert(CH > 0);
        const float ref = anchor(m);
        char* to = (char*)(out + sp.cut.head);
        auto one = [&](vec raw, int i) {
            const auto v = widened<T>(raw);
            typename Chunk<T>::wide g;
#pragma unroll
            for (int e = 0; e < E; ++e) g[e] = slope_at<ENT>(v[e], ref, c, A, B);
            __builtin_nontemporal_store(__builtin_convertvector(g, vec), (any*)(to + (size_t)(unsigned)i * 16));
        };
        const int j = sp.single();
        if (j >= 0) out[j] = (T)(slope_at<ENT>(alone, ref, c, A, B) + (j == y ? mark : 0.0f));
        const int t = thread();
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int i = sp.keep + k * BLOCK + t;
            if (in(k, i, sp.again, sp.end)) one(opaque(slot[k]), i);
            if (!HELD && sp.repeats()) fetch(sp, k, sp.origin, sp.begin, sp.again, t);
        }
        if constexpr (HELD) {
            for (int i = sp.origin + t; i < sp.again; i += BLOCK)       // (each thread its own: no barrier)
                if (i >= sp.begin) one(held[i - sp.origin], i);
        } else if (sp.repeats()) {
            for (int from = sp.origin; from < sp.again; from += BLOCK * CH) {
                const int on = from + BLOCK * CH;
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    const int i = from + k * BLOCK + t;
                    if (in(k, i, sp.begin, sp.again)) one(slot[k], i);
                    if (on < sp.again) fetch(sp, k, on, sp.begin, sp.again, t);
                }
            }
        }
        // the label's entry once more, by the thread that wrote its chunk
        const int i = (y - sp.cut.head) / E;
        if (y >= sp.cut.head && i >= sp.begin && i < sp.end && ((i - (i < sp.again ? sp.origin : sp.keep)) & (BLOCK - 1)) == (int)threadIdx.x)
            out[y] = (T)(slope_at<ENT>(zy, ref, c, A, B) + mark);
    }

    // zeros in a row, or piece `piece` of `pieces` of it
    static __device__ __forceinline__ void clear(T* out, int vocab, int piece = 0, int pieces = 1) {
        const Cut<T> cut(out, vocab);
        vec v;
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = (T)0.0f;
        for (int i = piece * BLOCK + (int)threadIdx.x - cut.lead(out); i < cut.whole; i += pieces * BLOCK)
            if (i >= 0) __builtin_nontemporal_store(v, (any*)((char*)(out + cut.head) + (size_t)(unsigned)i * 16));
        const int j = piece == 0 ? cut.single((int)threadIdx.x) : -1;
        if (j >= 0) out[j] = (T)0.0f;
    }
};

// ---- token log-probabilities -------------------------------------------------------------------------------------------

__device__ __forceinline__ float logp_of(Stat st, const RowLog& g, double s, float zy) {
    // (zy is no number where the label is past the vocabulary)
    return st.s == 0.0f ? (zy == zy ? -INFINITY : zy) : (float)(((double)zy - (double)st.m) * s - g.log_s);
}
template <typename T>
__device__ __forceinline__ float label_logit(const T* row, int64_t y, int vocab) {
    return y < vocab ? (float)row[y] : NAN;
}

__device__ __forceinline__ void put_token(const LogitsArgs& l, const TokenArgs& a, int64_t r, Stat st, float zy) {
    const RowLog g = row_log(st, l.s);
    const float lse = (float)g.lse;
    a.logp[r] = logp_of(st, g, l.s, zy);
    a.lse[r] = lse;
    // (past the end of 32 bits lse has taken it all)
    if (a.lse_rest)
        a.lse_rest[r] = fabsf(lse) < INFINITY ? (float)(((double)st.m * l.s - (double)lse) + g.log_s)
                                              : (fabs(g.lse) < INFINITY ? lse : 0.0f);
    if (a.entropy) a.entropy[r] = (float)g.entropy;
    if (a.top) {
        a.top[r] = st.m;
        a.sum[r] = st.s;
    }
}
__device__ __forceinline__ void put_no_token(const TokenArgs& a, int64_t r) {
    a.logp[r] = 0.0f;
    a.lse[r] = 0.0f;
    if (a.lse_rest) a.lse_rest[r] = 0.0f;
    if (a.entropy) a.entropy[r] = 0.0f;
    if (a.top) a.top[r] = a.sum[r] = 0.0f;
}

// One workgroup a row.  16400 x 131072 bf16 with the entropy 659 us: 6.5 TB/s of logits; 8 x 32768 5.8 us, most of it the launch and two
// trips to memory (label, then logits).
template <typename T, bool ENT, int BLOCK, int SLOTS>
__global__ __launch_bounds__(BLOCK) void k_token_logprob(LogitsArgs l, TokenArgs a, int64_t first) {
    __shared__ Stat lds[BLOCK / 64];
    const int64_t r = first + blockIdx.x;
    const T* row = (const T*)l.z + r * l.ld;
    const int64_t y = a.labels[r];
    if (y < 0) {
        if (threadIdx.x == 0) put_no_token(a, r);
        return;
    }
    typedef Row<T, BLOCK, 0, true, false, (BLOCK <= 512), SLOTS> Hold;
    const typename Hold::Span span(row, l.vocab);
    Hold z;
    z.open(span);
    const float zy = label_logit(row, y, l.vocab);
    const Stat st = block_stat<ENT, BLOCK / 64>(z.template stat<ENT, false>(span, l.c, nullptr), l.c, lds);
    if (threadIdx.x == 0) put_token(l, a, r, st, zy);
}

// What the way back knows of a row: p_j = 2^((z_j - ref) c) / sum, sum 0: the row has no distribution.
struct RowShare {
    float ref, sum;
};
__device__ __forceinline__ RowShare row_share(const LogitsArgs& l, const TokenGradArgs& a, int64_t r) {
    if (a.top) return {anchor(a.top[r]), a.sum[r]};
    // lse = ref s + off, ref the logit nearest to it.  Of lse_rest, which is known to 2^-25 of itself, more than 2^10 would leave off
    // uncertain by 2^-15 and more (lse is beyond 2^34 then, its own digits do not reach ln sum); then p_j is no number.
    const double lse = (double)a.lse[r], rest = a.lse_rest ? (double)a.lse_rest[r] : 0.0;
    const float ref = fminf(fmaxf((float)(lse * a.temperature), -FLT_MAX), FLT_MAX);
    if (lse == -INFINITY && rest == 0.0) return {ref, 0.0f};
    const double off = fma(-(double)ref, l.s, lse) + rest;
    return {ref, fabs(rest) <= 1024.0 && fabs(off) <= 80.0 ? exp2_hw((float)off * 1.44269504088896340736f) : NAN};
}

// The way back needs no sums: the forward call's do.  (From differences to the maximum, not as z_j s - lse: at a temperature that is no power of
// two the rounding of s takes all digits of that in a row far from 0.)  Workgroups take pieces of kGradChunks chunks a thread, one behind the other in
// memory, which is the kindest order to it: 8192 x 131072 bf16 690 us, 6.2 TB/s read and written.  (256 threads of four chunks each,
// us a preference step on 8192 x 131072, log-probabilities and all: 1100; 512 of two 1055, with loads past the caches 1027.)
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
    const int i0 = piece * (kGradBlock * kGradChunks) + (int)threadIdx.x - cut.lead(row);
    const int j = piece == 0 ? cut.single((int)threadIdx.x) : -1;
    const int64_t y = a.labels[r];
    const RowShare row_of = row_share(l, a, r);
    const float s = (float)l.s;
    // (a row without a distribution, a label of none: no gradient; a label past the vocabulary: no number)
    const bool none = y < 0 || row_of.sum == 0.0f;
    const float g = none ? 0.0f : (y < l.vocab ? a.d_logp[r] : NAN);
    const float h = !ENT || none ? 0.0f : a.d_entropy[r], entropy = !ENT || none ? 0.0f : a.entropy[r];
    if (g == 0.0f && h == 0.0f) {
        vec zero;
#pragma unroll
        for (int e = 0; e < E; ++e) zero[e] = (T)0.0f;
#pragma unroll
        for (int k = 0; k < kGradChunks; ++k)
            if (i0 + k * kGradBlock >= 0 && i0 + k * kGradBlock < cut.whole) *(any*)(to + (size_t)(unsigned)(i0 + k * kGradBlock) * 16) = zero;
        if (j >= 0) out[j] = (T)0.0f;
        return;
    }
    vec slot[kGradChunks];
#pragma unroll
    for (int k = 0; k < kGradChunks; ++k)
        if (i0 + k * kGradBlock >= 0 && i0 + k * kGradBlock < cut.whole) slot[k] = __builtin_nontemporal_load((const any*)(from + (size_t)(unsigned)(i0 + k * kGradBlock) * 16));
    // p_j (-g - h (log p_j + H)),  log p_j = ln 2 a_j - ln sum
    const float over = s / row_of.sum;
    const float log_sum = 0.693147180559945309417f * __builtin_amdgcn_logf(row_of.sum);      // (to 1e-6: every thread works it out)
    const float A = over * (ENT ? fmaf(h, log_sum - entropy, -g) : -g), B = over * -h * 0.693147180559945309417f;
    auto at = [&](float z) { return slope_at<ENT>(z, row_of.ref, l.c, A, B); };
    if (j >= 0) out[j] = (T)(at((float)row[j]) + (j == y ? g * s : 0.0f));
#pragma unroll
    for (int k = 0; k < kGradChunks; ++k) {
        const int i = i0 + k * kGradBlock;
        if (i < 0 || i >= cut.whole) continue;
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

// Everything about a row of the policy loss but its gradient's entries: dz_j = 2^a_j (A + B a_j), and `mark` more at the label.
struct PolicyRow {
    float loss, logp, entropy, A, B, mark;
    bool empty;
};
// dz_j = W (slope (1[j = y] - p_j) + c_H p_j (log p_j + H)),  log p_j = ln 2 a_j - ln S
template <bool ENT>
__device__ __forceinline__ PolicyRow policy_row(const LogitsArgs& l, const PolicyArgs& a, int64_t r, float w, Stat st, float zy) {
    const RowLog g = row_log(st, l.s);
    PolicyRow p;
    p.empty = st.s == 0.0f;
    p.logp = logp_of(st, g, l.s, zy);
    p.entropy = (float)g.entropy;
    const TokenLoss t = policy_token(a, r, p.logp);
    p.loss = ENT ? fmaf(-a.entropy_coef, p.entropy, t.loss) : t.loss;
    const float W = (float)((double)w * a.scale * l.s), over = W / st.s;
    p.A = over * (ENT ? fmaf(a.entropy_coef, (float)(g.entropy - g.log_s), -t.slope) : -t.slope);
    p.B = ENT ? over * a.entropy_coef * 0.693147180559945309417f : 0.0f;
    p.mark = W * t.slope;
    if (p.empty) p.A = p.B = p.mark = 0.0f;
    return p;
}
__device__ __forceinline__ void put_policy(const PolicyArgs& a, int64_t r, float loss, float logp, float entropy) {
    a.row_loss[r] = loss;
    a.logp[r] = logp;
    if (a.entropy) a.entropy[r] = entropy;
}

// One read and one write of the row.  8192 x 131072 bf16 788 us, 5.5 TB/s, 8192 x 65536 385 us, 5.6 TB/s, where copies of rows of the same
// shape through registers, without arithmetic, take 735 and 365: what is left is the time between a row's last load and its first
// store that the other workgroups of the compute unit do not fill.
template <typename T, bool ENT, int BLOCK, int CH, bool LONG, bool HELD>
__global__ __launch_bounds__(BLOCK, BLOCK == 512 ? 4 : 1) void k_policy(LogitsArgs l, PolicyArgs a, int64_t first) {
    typedef Row<T, BLOCK, CH, LONG, HELD> Hold;
    __shared__ Stat lds[BLOCK / 64];
    extern __shared__ __align__(16) unsigned char dyn[];
    const int64_t r = first + blockIdx.x, y = a.labels[r];
    const float w = a.weight ? a.weight[r] : 1.0f;
    T* out = (T*)l.dz + r * l.ld_dz;
    if (y < 0 || w == 0.0f) {
        if (threadIdx.x == 0) put_policy(a, r, 0.0f, 0.0f, 0.0f);
        Hold::clear(out, l.vocab);
        return;
    }
    const typename Hold::Span span((const T*)l.z + r * l.ld, l.vocab);
    Hold z;
    z.held = (typename Hold::vec*)dyn;
    z.open(span);
    const float zy = label_logit(span.row, y, l.vocab);
    const Stat st = block_stat<ENT, BLOCK / 64>(z.template stat<ENT, false>(span, l.c, nullptr), l.c, lds);
    const PolicyRow p = policy_row<ENT>(l, a, r, w, st, zy);
    if (threadIdx.x == 0) put_policy(a, r, p.loss, p.logp, p.entropy);
    z.template write<ENT>(span, out, st.m, l.c, p.A, p.B, y < l.vocab ? (int)y : -1, zy, p.mark);
}

// The same without a gradient.
template <typename T, bool ENT, int BLOCK, int SLOTS>
__global__ __launch_bounds__(BLOCK) void k_policy_value(LogitsArgs l, PolicyArgs a, int64_t first) {
    __shared__ Stat lds[BLOCK / 64];
    const int64_t r = first + blockIdx.x;
    const int64_t y = a.labels[r];
    const float w = a.weight ? a.weight[r] : 1.0f;
    if (y < 0 || w == 0.0f) {
        if (threadIdx.x == 0) put_policy(a, r, 0.0f, 0.0f, 0.0f);
        return;
    }
    typedef Row<T, BLOCK, 0, true, false, (BLOCK <= 512), SLOTS> Hold;
    const typename Hold::Span span((const T*)l.z + r * l.ld, l.vocab);
    Hold z;
    z.open(span);
    const float zy = label_logit(span.row, y, l.vocab);
    const Stat st = block_stat<ENT, BLOCK / 64>(z.template stat<ENT, false>(span, l.c, nullptr), l.c, lds);
    const PolicyRow p = policy_row<ENT>(l, a, r, w, st, zy);
    if (threadIdx.x == 0) put_policy(a, r, p.loss, p.logp, p.entropy);
}

// ---- distillation ----------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float teacher_logit(const DistillArgs& a, int64_t at) {
    return a.logit_type == LBFGSB_F32 ? ((const float*)a.logit)[at]
         : a.logit_type == LBFGSB_BF16 ? (float)((const __bf16*)a.logit)[at] : (float)((const _Float16*)a.logit)[at];
}
__device__ __forceinline__ int64_t teacher_index(const DistillArgs& a, int64_t at) {
    return a.index_type == LBFGSB_I32 ? (int64_t)((const int*)a.index)[at] : ((const int64_t*)a.index)[at];
}

// LDS of the distillation kernel: a row's entries (index, teacher's share, student's logit, scratch), then one bit for each
// entry of the vocabulary.
struct TopLds {
    int* at;
    float *q, *z, *scratch;
    unsigned* seen;
};
__device__ __forceinline__ TopLds top_lds(unsigned char* dyn, int top) {
    TopLds s;
    s.at = (int*)dyn;
    s.q = (float*)(s.at + top);
    s.z = s.q + top;
    s.scratch = s.z + top;
    s.seen = (unsigned*)(s.scratch + top);
    return s;
}
__host__ __device__ inline size_t distill_lds(int top, int vocab) { return (size_t)top * 16 + (size_t)(vocab + 8 + 127) / 128 * 16; }

// Between an LDS write of one lane and a read by another of the same wave.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <int BLOCK>
__device__ __forceinline__ void clear_seen(TopLds s, int vocab) {
    for (int i = threadIdx.x; i < (vocab + 8 + 127) / 128 * 4; i += BLOCK) s.seen[i] = 0;
    __syncthreads();
}

struct Marks {
    bool lost, twice;       // of this lane's entries: past the vocabulary, a second time
};
// By the first wave: the entries' indices (-1: padding) and the teacher's logits into LDS, and the indices' bits in `seen`, `by` further on.
// REST: all bits are zero before; else the words in question are cleared here.
template <bool REST>
__device__ __forceinline__ Marks mark_entries(const LogitsArgs& l, const DistillArgs& a, int64_t r, int by, TopLds s) {
    Marks m{false, false};
    for (int k = threadIdx.x; k < a.top; k += 64) {
        const int64_t j = teacher_index(a, r * a.ld + k);
        const float v = teacher_logit(a, r * a.ld + k);
        m.lost |= j >= l.vocab;
        const bool none = j < 0 || j >= l.vocab || v == -INFINITY;
        s.at[k] = none ? -1 : (int)j;
        s.q[k] = v;
        if (!REST && !none) s.seen[((int)j + by) >> 5] = 0;
    }
    wave_fence();
    for (int k = threadIdx.x; k < a.top; k += 64)
        if (s.at[k] >= 0) {
            const int place = s.at[k] + by;
            const unsigned bit = 1u << (place & 31);
            m.twice |= (atomicOr(&s.seen[place >> 5], bit) & bit) != 0;
        }
    return m;
}

// By the first wave, after mark_entries: the entries' shares (an index that comes twice keeps its first place only, with the sum of its
// shares), the student's logits there and what all of them come to.  REST: the student's statistics over the entries as well.
template <typename T, bool REST>
__device__ __forceinline__ void read_teacher(const LogitsArgs& l, const DistillArgs& a, int64_t r, const T* row, Marks marks, TopLds s,
                                             Teacher* out) {
    const int lane = threadIdx.x & 63, top = a.top;
    float most = -INFINITY, z_top = -INFINITY;
    for (int k = lane; k < top; k += 64) {
        s.z[k] = s.at[k] >= 0 ? (float)row[s.at[k]] : -INFINITY;
        z_top = fmaxf(z_top, s.z[k]);
        if (s.at[k] >= 0) most = fmaxf(most, s.q[k]);
    }
    wave_fence();
    most = lane_bcast_f(anchor(wave_max_f(most)), 0);
    z_top = lane_bcast_f(anchor(wave_max_f(z_top)), 0);      // (in a scalar register)
    // with e_k = exp(s (a_k - most)):  sums of e, e (a - most), e (z - z_top), and of nothing else, so that one reduction does.
    // (Differences to the largest: of a row at the type's lowest value sums of the logits themselves would leave no digit.)
    double sums[8] = {};
    for (int k = lane; k < top; k += 64) {
        if (s.at[k] < 0) continue;
        const float d = s.q[k] - most, e = exp2_hw(d * l.c.c);
        s.q[k] = e;
        sums[0] += (double)e;
        if (e != 0.0f) {
            sums[1] = fma((double)e, (double)d, sums[1]);
            float from = z_top;
            asm volatile("" : "+s"(from));            // (widened here, not kept in two more registers)
            sums[2] = fma((double)e, (double)s.z[k] - (double)from, sums[2]);
        }
    }
    wave_fence();
    if (__any(marks.twice)) {
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
    const double mine = wave_sums8(sums, lane);
    const double total = lane_bcast(mine, 0), ed = lane_bcast(mine, 1), ez = lane_bcast(mine, 2);
    // q_k = f e_k and log q_k = s (a_k - most) - shift
    double f, shift;
    if (total == 0.0) {               // no entry, whatever the log-sum-exp is
        f = shift = 0.0;
    } else if (a.lse) {
        shift = (double)a.lse[r] - (double)most * l.s;
        f = (double)expf((float)-shift);
    } else {
        shift = total > 0.0 ? log_d(total) : total;
        f = 1.0 / total;
    }
    Running run;
    int entries = 0;
    for (int k0 = 0; k0 < top; k0 += 64) {
        const int k = k0 + lane;
        const bool one = k < top && s.at[k] >= 0;
        entries += __popcll(__ballot(one));
        if (!one) continue;
        s.q[k] = (float)(f * (double)s.q[k]);
        if (REST) {
            const float v[1] = {s.z[k]};
            run.take<false>(v, l.c);
        }
    }
    const Stat st = REST ? wave_stat<false>(run.a, l.c) : run.a;
    const int any_lost = __any(marks.lost);
    if (lane == 0) *out = {f * (l.s * (ed - ez) - shift * total), f * total, z_top, st, entries, any_lost};
}

// What a row of the distillation's gradient is made of: away from the teacher's dz_j = A 2^((z_j - st.m) c), at one of them
// W (p_j - q_j).  st: over the row, REST: over what is not among the entries; all: over the row.
struct DistillRow {
    Stat all;
    float A, W;
    bool empty;
    __device__ __forceinline__ float at_entry(float z, float q, Factor c) const {
        return W * (exp2_hw((z - anchor(all.m)) * c.c) / all.s - q);
    }
};
// the teacher's share of the rest
__device__ __forceinline__ double teacher_rest(const LogitsArgs& l, const Teacher& t) {
    return t.entries < l.vocab && t.sum < 1.0 ? 1.0 - t.sum : 0.0;
}
template <bool REST>
__device__ __forceinline__ DistillRow distill_row(const LogitsArgs& l, const DistillArgs& a, float w, Stat st, const Teacher& t) {
    DistillRow d;
    d.all = REST ? merged(st, t.top, l.c) : st;
    d.empty = (d.all.s == 0.0f || !t.entries) && !t.lost;
    // (a teacher that is no number leaves its mark on every entry)
    d.W = t.lost || t.cross != t.cross ? NAN : (float)((double)w * a.scale * l.s);
    if (REST) {
        // p_j (1 - r / t), the student's share t = sum over the rest / sum over the row
        const double share = (double)(st.s * exp2_hw(below(st.m, d.all.m, l.c)) / d.all.s);
        d.A = st.s == 0.0f ? 0.0f : d.W * (float)((share - teacher_rest(l, t)) / (double)st.s);
    } else {
        d.A = d.W / st.s;
    }
    return d;
}
template <bool REST>
__device__ __forceinline__ float distill_value(const LogitsArgs& l, Stat st, const Teacher& t) {
    const Stat all = REST ? merged(st, t.top, l.c) : st;
    if (t.lost) return NAN;
    if (!t.entries) return 0.0f;
    if (all.s == 0.0f) return INFINITY;
    const RowLog g = row_log(all, l.s);
    asm volatile("" ::: "memory");            // (the rest of t is read now, not kept through the logarithm)
    double loss = t.cross + t.sum * (((double)all.m - (double)t.z_top) * l.s + g.log_s);
    if (REST) {
        const double rest = teacher_rest(l, t);
        const double log_t = st.s == 0.0f ? -INFINITY : ((double)st.m - (double)all.m) * l.s + log_d((double)st.s) - g.log_s;
        if (rest > 0.0) loss += rest * (log_d(rest) - log_t);
    }
    return (float)loss;
}

// As the policy loss, and the first wave looks after the teacher meanwhile: its entries, then the student's logits there, one more trip
// to memory, and two dozen double sums.  8192 x 65536 bf16, 64 entries, 400 us, 5.4 TB/s; with the rest's outcome, which has to know
// the entries before the statistics, 415.  (With the entries loaded ahead of the row's chunks
// it is no faster: 842 / 862 us at 8192 x 131072.)
template <typename T, bool REST, int BLOCK, int CH, bool LONG, bool HELD>
__global__ __launch_bounds__(BLOCK, BLOCK == 512 ? 4 : 1) void k_distill(LogitsArgs l, DistillArgs a, int64_t first) {
    __shared__ Stat lds[BLOCK / 64];
    __shared__ Teacher teacher;
    extern __shared__ __align__(16) unsigned char dyn[];
    const TopLds s = top_lds(dyn, a.top);
    const int64_t r = first + blockIdx.x;
    const T* row = (const T*)l.z + r * l.ld;
    T* out = (T*)l.dz + r * l.ld_dz;
    const float w = a.weight ? a.weight[r] : 1.0f;
    if (w == 0.0f) {
        if (threadIdx.x == 0) a.row_loss[r] = 0.0f;
        if (l.dz) Row<T, BLOCK, CH>::clear(out, l.vocab);
        return;
    }
    typedef Row<T, BLOCK, CH, LONG, HELD> Hold;
    const typename Hold::Span span(row, l.vocab);
    Hold z;
    z.held = (typename Hold::vec*)(dyn + distill_lds(a.top, l.vocab));
    z.open(span);
    if (REST) clear_seen<BLOCK>(s, l.vocab);
    Marks marks{false, false};
    if (threadIdx.x < 64) marks = mark_entries<REST>(l, a, r, span.cut.shift(), s);
    if (REST) __syncthreads();
    if (threadIdx.x < 64) read_teacher<T, REST>(l, a, r, row, marks, s, &teacher);
    const Stat st = block_stat<false, BLOCK / 64>(z.template stat<false, REST>(span, l.c, (const unsigned char*)s.seen), l.c, lds);
    const DistillRow d = distill_row<REST>(l, a, w, st, teacher);
    if (threadIdx.x == 0) a.row_loss[r] = distill_value<REST>(l, st, teacher);
    if (!l.dz) return;
    if (d.empty) {
        Row<T, BLOCK, CH>::clear(out, l.vocab);
        return;
    }
    z.template write<false>(span, out, st.m, l.c, d.A, 0.0f, -1, 0.0f, 0.0f);
    __syncthreads();                          // (the entries' own values come after the row's)
    for (int k = threadIdx.x; k < a.top; k += BLOCK)
        if (s.at[k] >= 0) out[s.at[k]] = (T)d.at_entry(s.z[k], s.q[k], l.c);
}

// ---- a few long rows, in pieces ----------------------------------------------------------------------------------------------
// One workgroup a row leaves most of the chip idle when there are few: the statistics of a row's pieces by a workgroup each, then, in
// a second launch, the join and the gradient by as many.  (The second reads the logits again, out of the caches.)  Each of the two
// takes about 4 us at 16 x 32768 f32, as long as a launch that does nothing but load once and store.

constexpr int kSplitBlock = 512, kSplitHold = 4;      // threads; chunks a thread holds in the second launch

// the statistics of a row, by every wave of the second launch
template <bool ENT>
__device__ __forceinline__ Stat joined(const SplitRow& s, int splits, Factor c) {
    const int lane = threadIdx.x & 63;
    return wave_stat<ENT>(lane < splits ? s.part[lane] : Stat{-INFINITY, 0.0f, 0.0f}, c);
}
// the same by one lane
__device__ __forceinline__ Stat joined_alone(const SplitRow& s, int splits, Factor c) {
    Stat a = s.part[0];
    for (int i = 1; i < splits; ++i) a = merged(a, s.part[i], c);
    return a;
}

template <typename T, bool ENT>
__global__ __launch_bounds__(kSplitBlock) void k_split(LogitsArgs l, const int64_t* labels, const float* weight, SplitRow* ws, int splits) {
    __shared__ Stat lds[kSplitBlock / 64];
    const int r = blockIdx.x / splits, i = blockIdx.x % splits;
    const T* row = (const T*)l.z + r * l.ld;
    const int64_t y = labels[r];
    if (y < 0 || (weight && weight[r] == 0.0f)) return;
    typedef Row<T, kSplitBlock, 0, true, false, false> Hold;
    const typename Hold::Span span(row, l.vocab, i, splits);
    Hold z;
    z.open(span);
    const float zy = label_logit(row, y, l.vocab);
    const Stat st = block_stat<ENT, kSplitBlock / 64>(z.template stat<ENT, false>(span, l.c, nullptr), l.c, lds);
    if (threadIdx.x == 0) {
        ws[r].part[i] = st;
        if (i == 0) ws[r].zy = zy;            // (the second launch may write the gradient over it)
    }
}

// One workgroup more for each row: the teacher's entries.
template <typename T, bool REST>
__global__ __launch_bounds__(kSplitBlock) void k_split_distill(LogitsArgs l, DistillArgs a, SplitRow* ws, int splits) {
    __shared__ Stat lds[kSplitBlock / 64];
    extern __shared__ __align__(16) unsigned char dyn[];
    const TopLds s = top_lds(dyn, a.top);
    const int r = blockIdx.x / (splits + 1), i = blockIdx.x % (splits + 1);
    const T* row = (const T*)l.z + r * l.ld;
    if (a.weight && a.weight[r] == 0.0f) return;
    if (i == splits) {
        const Cut<T> cut(row, l.vocab);
        if (REST) clear_seen<kSplitBlock>(s, l.vocab);
        if (threadIdx.x < 64) read_teacher<T, REST>(l, a, r, row, mark_entries<REST>(l, a, r, cut.shift(), s), s, &ws[r].teacher);
        __syncthreads();
        for (int k = threadIdx.x; k < a.top; k += kSplitBlock) {
            ws[r].at[k] = s.at[k];
            ws[r].q[k] = s.q[k];
            ws[r].z[k] = s.z[k];
        }
        return;
    }
    typedef Row<T, kSplitBlock, 0, true, false, false> Hold;
    const typename Hold::Span span(row, l.vocab, i, splits);
    Hold z;
    z.open(span);
    if (REST) {
        clear_seen<kSplitBlock>(s, l.vocab);
        for (int k = threadIdx.x; k < a.top; k += kSplitBlock) {
            const int64_t j = teacher_index(a, r * a.ld + k);
            if (j >= 0 && j < l.vocab && teacher_logit(a, r * a.ld + k) != -INFINITY)
                atomicOr(&s.seen[((int)j + span.cut.shift()) >> 5], 1u << (((int)j + span.cut.shift()) & 31));
        }
        __syncthreads();
    }
    const Stat st = block_stat<false, kSplitBlock / 64>(z.template stat<false, REST>(span, l.c, (const unsigned char*)s.seen), l.c, lds);
    if (threadIdx.x == 0) ws[r].part[i] = st;
}

__global__ __launch_bounds__(64) void k_join_token(LogitsArgs l, TokenArgs a, const SplitRow* ws, int splits) {
    const int r = blockIdx.x;
    if (a.labels[r] < 0) {
        if (threadIdx.x == 0) put_no_token(a, r);
        return;
    }
    const Stat st = joined<true>(ws[r], splits, l.c);
    if (threadIdx.x == 0) put_token(l, a, r, st, ws[r].zy);
}

// The last workgroup of the second launch has the total, a lane for each row.
__device__ __forceinline__ void put_total(double mine, double scale, float* loss) {
    const double sum = wave_sum(mine);
    if (threadIdx.x == 0) *loss = (float)(sum * scale);
}

template <typename T, bool ENT>
__global__ __launch_bounds__(kSplitBlock) void k_join_policy(LogitsArgs l, PolicyArgs a, const SplitRow* ws, int splits, float* loss) {
    const int r = blockIdx.x / splits, i = blockIdx.x % splits;
    if (r == l.rows) {
        if (threadIdx.x >= 64) return;
        const int q = threadIdx.x;
        const float w = q < l.rows ? (a.weight ? a.weight[q] : 1.0f) : 0.0f;
        double mine = 0.0;
        if (w != 0.0f && a.labels[q] >= 0)
            mine = (double)w * (double)policy_row<ENT>(l, a, q, w, joined_alone(ws[q], splits, l.c), ws[q].zy).loss;
        put_total(mine, a.scale, loss);
        return;
    }
    T* out = (T*)l.dz + r * l.ld_dz;
    const int64_t y = a.labels[r];
    const float w = a.weight ? a.weight[r] : 1.0f;
    if (y < 0 || w == 0.0f) {
        if (threadIdx.x == 0 && i == 0) put_policy(a, r, 0.0f, 0.0f, 0.0f);
        if (l.dz) Row<T, kSplitBlock, kSplitHold>::clear(out, l.vocab, i, splits);
        return;
    }
    typedef Row<T, kSplitBlock, kSplitHold, true> Hold;
    const typename Hold::Span span((const T*)l.z + r * l.ld, l.vocab, i, splits);
    Hold z;
    z.open_last(span);
    const Stat st = joined<ENT>(ws[r], splits, l.c);
    const PolicyRow p = policy_row<ENT>(l, a, r, w, st, ws[r].zy);
    if (threadIdx.x == 0 && i == 0) put_policy(a, r, p.loss, p.logp, p.entropy);
    if (!l.dz) return;
    if (p.empty) Row<T, kSplitBlock, kSplitHold>::clear(out, l.vocab, i, splits);
    else z.template write<ENT>(span, out, st.m, l.c, p.A, p.B, y < l.vocab ? (int)y : -1, ws[r].zy, p.mark);
}

template <typename T, bool REST>
__global__ __launch_bounds__(kSplitBlock) void k_join_distill(LogitsArgs l, DistillArgs a, const SplitRow* ws, int splits, float* loss) {
    const int r = blockIdx.x / splits, i = blockIdx.x % splits;
    if (r == l.rows) {
        if (threadIdx.x >= 64) return;
        const int q = threadIdx.x;
        const float w = q < l.rows ? (a.weight ? a.weight[q] : 1.0f) : 0.0f;
        double mine = 0.0;
        if (w != 0.0f) mine = (double)w * (double)distill_value<REST>(l, joined_alone(ws[q], splits, l.c), ws[q].teacher);
        put_total(mine, a.scale, loss);
        return;
    }
    T* out = (T*)l.dz + r * l.ld_dz;
    const float w = a.weight ? a.weight[r] : 1.0f;
    if (w == 0.0f) {
        if (threadIdx.x == 0 && i == 0) a.row_loss[r] = 0.0f;
        if (l.dz) Row<T, kSplitBlock, kSplitHold>::clear(out, l.vocab, i, splits);
        return;
    }
    typedef Row<T, kSplitBlock, kSplitHold, true> Hold;
    const typename Hold::Span span((const T*)l.z + r * l.ld, l.vocab, i, splits);
    Hold z;
    z.open_last(span);
    const Stat st = joined<false>(ws[r], splits, l.c);
    const DistillRow d = distill_row<REST>(l, a, w, st, ws[r].teacher);
    if (threadIdx.x == 0 && i == 0) a.row_loss[r] = distill_value<REST>(l, st, ws[r].teacher);
    if (!l.dz) return;
    if (d.empty) {
        Row<T, kSplitBlock, kSplitHold>::clear(out, l.vocab, i, splits);
        return;
    }
    z.template write<false>(span, out, st.m, l.c, d.A, 0.0f, -1, 0.0f, 0.0f);
    __syncthreads();                          // (the entries' own values come after the row's)
    for (int k = threadIdx.x; k < a.top; k += kSplitBlock) {
        const int j = ws[r].at[k];
        if (j >= 0 && span.has(j)) out[j] = (T)d.at_entry(ws[r].z[k], ws[r].q[k], l.c);
    }
}

// how many places of a chunk a row takes, at most, with those before its first that bring it to a line
template <typename T>
int most_chunks(const LogitsArgs& l) {
    const bool lines = ((uintptr_t)l.z & 127) == 0 && l.ld * (int64_t)sizeof(T) % 128 == 0;
    return l.vocab / Chunk<T>::E + (lines ? 0 : 7);
}

// f(first row or piece, workgroups) for each launch
template <typename F>
void by_rows(int64_t rows, F f) {
    for (int64_t r = 0; r < rows; r += kRowBlocksMax) f(r, dim3((unsigned)(rows - r < kRowBlocksMax ? rows - r : kRowBlocksMax)));
}

// f(BLOCK, SLOTS) for rows of `vocab` elements that are only read
template <typename T, typename F>
void by_length(int64_t rows, int vocab, F f) {
    // Where there are rows for every compute unit, few threads to each; where there are not, many.  bf16, us, 64 / 256 / 512 threads, two
    // loads each: 16384 x 2000 16.4 / 24.7 / 41, x 8000 45.7 / 48.0 / 58, x 32000 164 / 162 / 163, 3001 x 50021 (f16) 54 / 53 / 47;
    // 512 and 1024 threads, four loads: 128 x 4000 4.3 (64 threads) / 3.4 (512), 128 x 32768 6.5 (256) / 4.8 (1024).
    const int chunks = vocab / Chunk<T>::E;
    using std::integral_constant;
    if (rows <= 512) {
        if (chunks <= 1024) f(integral_constant<int, 512>{}, integral_constant<int, 4>{});
        else f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    } else {
        if (chunks <= 1024) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
        else if (chunks <= 4096) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
        else f(integral_constant<int, 512>{}, integral_constant<int, 2>{});
    }
}

// LDS of what a row of `chunks` places has before the HOLD - 16 that stay in registers (Span), and what each of two workgroups of a compute
// unit may have of it.
inline size_t held_bytes(int chunks, int hold) { return (size_t)(chunks - (hold - 16) + 16) * 16; }
constexpr size_t kPairLds = 79 << 10;

// f(BLOCK, CH, LONG, HELD) for rows whose gradient is wanted: the fewest threads whose registers hold the row, 4 to 16 chunks each, since several
// small workgroups on a compute unit fill each other's pauses.  Policy loss, 16384 rows of bf16, us: x 1000 64 threads of 4 chunks 27, 128 of 4
// 34, 256 of 4 47; x 4000 128 of 4 61, 256 of 4 64, 512 of 4 91; x 8000 256 of 4 99, 512 of 4 121; x 16000 256 of 8 193, 512 of 4 188 (the
// distillation 209 and 242); x 32000 512 of 8 372, 256 of 16 no less.  Of 512 threads the count of chunks follows the row: 4099 x 50021 f16 13 chunks
// 135, 16 chunks 143.  Longer rows than 1024 threads hold: 1001 x 100003 f32 read twice 245, kept as far as it goes 184 (both from
// before loads went past the caches and chunks began on lines; 148 since).
// Rows of more than 8192 chunks: one workgroup of 1024 threads on a compute unit, or with many rows of 16 bits two of 512, of which one loads
// while the other writes, with 23 chunks a thread and what is left of the row in LDS (`lds` bytes of it are taken already).  1024 / 512
// threads, us, bf16.  In registers alone, policy loss x 70000: 128 rows 13.8 / 14.4, 400 29.9 / 23.5, 8192 473 / 400; x 92000, 400 rows
// 36.4 / 28.5, 8192 602 / 565.  With LDS, policy loss x 131072: 1000 rows 102 / 110, 1500 164 / 156, 4000 413 / 391, 8192 818 / 788; x 100000,
// 1000 rows 76 / 81, 8192 657 / 593.  Distillation with the rest, which spills at 512, x 80000: 1000 rows 78 / 89, 4000 315 / 288, 8192 635 / 556,
// and with LDS, x 100000, 8192 rows 747 / 777.  f32, policy loss, 4000 rows: x 50021 290 / 296, x 62003 352 / 363.
// PAIR, HELD: the rows from which it is two of 512 threads, in registers alone and with LDS (0: never): from where on the pair won at every count
// above.  (Between two of them how full the last round of 256 or 512 workgroups is decides, which these counts do not follow.)
template <typename T, int PAIR, int HELD, typename F>
void by_width(const LogitsArgs& l, size_t lds, F f) {
    const int chunks = most_chunks<T>(l);
    using std::integral_constant;
    constexpr std::false_type no{};
    constexpr std::true_type yes{};
    if (chunks <= 64 * 4) f(integral_constant<int, 64>{}, integral_constant<int, 4>{}, no, no);
    else if (chunks <= 128 * 4) f(integral_constant<int, 128>{}, integral_constant<int, 4>{}, no, no);
    else if (chunks <= 256 * 4) f(integral_constant<int, 256>{}, integral_constant<int, 4>{}, no, no);
    else if (chunks <= 256 * 8) f(integral_constant<int, 256>{}, integral_constant<int, 8>{}, no, no);
    else if (chunks <= 512 * 8) f(integral_constant<int, 512>{}, integral_constant<int, 8>{}, no, no);
    else if (chunks <= 512 * 10) f(integral_constant<int, 512>{}, integral_constant<int, 10>{}, no, no);
    else if (chunks <= 512 * 13) f(integral_constant<int, 512>{}, integral_constant<int, 13>{}, no, no);
    else if (chunks <= 512 * 16) f(integral_constant<int, 512>{}, integral_constant<int, 16>{}, no, no);
    else {
        if constexpr (PAIR > 0 && sizeof(T) == 2) {
            if (chunks <= 512 * 23 && l.rows >= PAIR) return f(integral_constant<int, 512>{}, integral_constant<int, 23>{}, no, no);
        }
        if constexpr (HELD > 0 && sizeof(T) == 2) {
            if (chunks > 512 * 23 && l.rows >= HELD && held_bytes(chunks, 512 * 23) + lds <= kPairLds)
                return f(integral_constant<int, 512>{}, integral_constant<int, 23>{}, yes, yes);
        }
        if (chunks <= 1024 * 13) f(integral_constant<int, 1024>{}, integral_constant<int, 13>{}, no, no);
        else if (chunks <= 1024 * 16) f(integral_constant<int, 1024>{}, integral_constant<int, 16>{}, no, no);
        else f(integral_constant<int, 1024>{}, integral_constant<int, 16>{}, yes, no);
    }
}

}  // namespace

// LDS beyond what a kernel has without asking
template <typename K>
hipError_t allow_lds(K kernel, size_t bytes) {
    if (bytes <= 60 << 10) return hipSuccess;
    return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T>
hipError_t token_logprob_rows(const LogitsArgs& l, const TokenArgs& a, SplitRow* ws, hipStream_t st) {
    if (const int splits = row_splits(l.rows, l.vocab, sizeof(T), false); splits > 1) {
        const auto kernel = a.entropy ? k_split<T, true> : k_split<T, false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.rows * splits), dim3(kSplitBlock), 0, st, l, a.labels, (const float*)nullptr, ws, splits);
        hipLaunchKernelGGL(k_join_token, dim3((unsigned)l.rows), dim3(64), 0, st, l, a, (const SplitRow*)ws, splits);
        return hipGetLastError();
    }
    by_length<T>(l.rows, l.vocab, [&](auto block, auto slots) {
        constexpr int BLOCK = decltype(block)::value, SLOTS = decltype(slots)::value;
        const auto kernel = a.entropy ? k_token_logprob<T, true, BLOCK, SLOTS> : k_token_logprob<T, false, BLOCK, SLOTS>;
        by_rows(l.rows, [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(BLOCK), 0, st, l, a, first); });
    });
    return hipGetLastError();
}

template <typename T>
hipError_t token_grad_rows(const LogitsArgs& l, const TokenGradArgs& a, hipStream_t st) {
    constexpr int kPiece = kGradBlock * kGradChunks;
    const int64_t pieces = (std::max(most_chunks<T>(l), 1) + kPiece - 1) / kPiece;      // (one for a row of single elements too)
    const auto kernel = a.d_entropy ? k_token_grad<T, true> : k_token_grad<T, false>;
    by_rows(l.rows * pieces,
            [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kGradBlock), 0, st, l, a, (int)pieces, first); });
    return hipGetLastError();
}

template <typename T>
hipError_t policy_rows(const LogitsArgs& l, const PolicyArgs& a, float* loss, SplitRow* ws, hipStream_t st) {
    const bool ent = a.entropy || a.entropy_coef != 0.0f;
    if (const int splits = row_splits(l.rows, l.vocab, sizeof(T), l.dz != nullptr); splits > 1) {
        const unsigned blocks = (unsigned)l.rows * splits;
        hipLaunchKernelGGL((ent ? k_split<T, true> : k_split<T, false>), dim3(blocks), dim3(kSplitBlock), 0, st, l, a.labels, a.weight, ws, splits);
        hipLaunchKernelGGL((ent ? k_join_policy<T, true> : k_join_policy<T, false>), dim3(blocks + 1), dim3(kSplitBlock), 0, st, l, a,
                           (const SplitRow*)ws, splits, loss);
        return hipGetLastError();
    }
    hipError_t err = hipSuccess;
    if (!l.dz) by_length<T>(l.rows, l.vocab, [&](auto block, auto slots) {
        constexpr int BLOCK = decltype(block)::value, SLOTS = decltype(slots)::value;
        const auto kernel = ent ? k_policy_value<T, true, BLOCK, SLOTS> : k_policy_value<T, false, BLOCK, SLOTS>;
        by_rows(l.rows, [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(BLOCK), 0, st, l, a, first); });
    });
    else if (ent) by_width<T, 0, 0>(l, 0, [&](auto block, auto ch, auto lng, auto) {
        constexpr int BLOCK = decltype(block)::value, CH = decltype(ch)::value;
        const auto kernel = k_policy<T, true, BLOCK, CH, decltype(lng)::value, false>;
        by_rows(l.rows, [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(BLOCK), 0, st, l, a, first); });
    });
    else by_width<T, 257, 1500>(l, 0, [&](auto block, auto ch, auto lng, auto held) {
        constexpr int BLOCK = decltype(block)::value, CH = decltype(ch)::value;
        const auto kernel = k_policy<T, false, BLOCK, CH, decltype(lng)::value, decltype(held)::value>;
        const size_t lds = decltype(held)::value ? held_bytes(most_chunks<T>(l), BLOCK * CH) : 0;
        err = allow_lds(kernel, lds);
        if (err != hipSuccess) return;
        by_rows(l.rows, [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(BLOCK), lds, st, l, a, first); });
    });
    if (err != hipSuccess) return err;
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    return launch_weighted_total(a.row_loss, a.weight, l.rows, a.scale, loss, st);
}

template <typename T>
hipError_t distill_rows(const LogitsArgs& l, const DistillArgs& a, float* loss, SplitRow* ws, hipStream_t st) {
    const size_t lds = distill_lds(a.top, l.vocab);
    if (const int splits = row_splits(l.rows, l.vocab, sizeof(T), l.dz != nullptr); splits > 1) {
        const auto kernel = a.lse ? k_split_distill<T, true> : k_split_distill<T, false>;
        if (hipError_t e = allow_lds(kernel, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)l.rows * (splits + 1)), dim3(kSplitBlock), lds, st, l, a, ws, splits);
        hipLaunchKernelGGL((a.lse ? k_join_distill<T, true> : k_join_distill<T, false>), dim3((unsigned)l.rows * splits + 1), dim3(kSplitBlock), 0,
                           st, l, a, (const SplitRow*)ws, splits, loss);
        return hipGetLastError();
    }
    hipError_t err = hipSuccess;
    auto launch = [&](auto rest, auto block, auto ch, auto lng, auto held) {
        constexpr int BLOCK = decltype(block)::value, CH = decltype(ch)::value;
        const auto kernel = k_distill<T, decltype(rest)::value, BLOCK, CH, decltype(lng)::value, decltype(held)::value>;
        const size_t more = decltype(held)::value ? held_bytes(most_chunks<T>(l), BLOCK * CH) : 0;
        err = allow_lds(kernel, lds + more);
        if (err != hipSuccess) return;
        by_rows(l.rows, [&](int64_t first, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(BLOCK), lds + more, st, l, a, first); });
    };
    if (a.lse) by_width<T, 4000, 0>(l, lds, [&](auto... w) { launch(std::true_type{}, w...); });
    else by_width<T, 257, 1500>(l, lds, [&](auto... w) { launch(std::false_type{}, w...); });
    if (err != hipSuccess || (err = hipGetLastError()) != hipSuccess) return err;
    return launch_weighted_total(a.row_loss, a.weight, l.rows, a.scale, loss, st);
}

}  // namespace lb
