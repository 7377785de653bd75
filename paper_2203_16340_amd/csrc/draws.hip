// Tokens drawn from rows of logits by given numbers, and drafted tokens verified against the target's rows.
//
// A token is the first entry at which the running sum of p passes u.  With e_j = 2^((z_j - ref) c) a row is read once, in blocks of
// 4 kB whose sums are kept (8 bytes a block: 0.2 % of the row); in 64 bits the blocks' sums tell the block in which u S is
// passed, S being the whole row's, and that block alone is read again, lane by lane and entry by entry.
// Exponentials, a block's sum and the weight that brings it to the row's largest are in 32 bits, sums over blocks, the walk and logarithms in 64.  With
// units of 2^-24: an exponent -a of 2 is off by 2.5 a ln 2 (difference, product, the factor's second part) and what lies there, of 2^21 entries at
// most, is 2^(21 - a) / (1 + 2^(21 - a)) of the row, so that S is off by 28 at most (a = 17 or 18); the two exponentials by 4, a block's sum of
// 2048 by 14: 46 units, 2.8e-6.  Measured, at a tail of equal entries that holds most of the row: borders 2.9e-7, log p 2.1e-6.
//
// Verification: the same sums tell whether a drafted token is accepted; where the first is not, blocks of max(p - q, 0) are summed and walked through
// alike.  A workgroup takes a request, position by position; few requests are taken in two launches, sums of all rows and then the rest, by many.
#include "draws.h"

namespace lb {

namespace {

constexpr int kDrawBlock = 256, kDrawWaves = kDrawBlock / 64;

// 2^((z - ref) c) as it enters the sums of blocks: c is the factor's first part alone, which is off by 2^-25 of the distance to the wave's largest so
// far, to one side (1e-8 of it at temperature 1); joins of blocks take both parts.  (Both at every entry: 1001 x 50021 f16 24.5 us for 21.6, 256
// requests of 5 drafts 101 for 93.)
__device__ __forceinline__ float share(float z, float ref, float c) { return exp2_hw((z - ref) * c); }
// 2^((z - ref) c + e), with the second parts of both, for differences p - q.  (Where z is the largest's equal or not far from it the first exponent is
// small, whatever its parts are, and so is its rounding.  The second takes no part where it is small against a distance without end.  With draft_logp the
// drafter's ref is the drafted token's logit, which may be far below the largest: what z - ref loses there is 2^-24 of the token's -log q.)
__device__ __forceinline__ float mass(float z, float ref, Factor c, Exponent e) {
    const float d = z - ref, x = exp2_hw(fmaf(d, c.c, e.high));
    return fmaf(x, fmaf(fmaxf(d, -1000.0f), c.low * 0.693147181f, e.low), x);
}
__device__ __forceinline__ Exponent exponent_of(double log) {       // of e to one of 2
    const double x = log * 1.44269504088896340736;
    return {(float)x, (float)((x - (double)(float)x) * 0.69314718055994530942)};
}

// A row as it is read in blocks: chunks of 16 bytes on boundaries of the logits, of which the first and the last may hold less of the row.
template <typename T>
struct Line {
    static constexpr int E = Chunk<T>::E, kPer = kBlockBytes / 16, kLoads = kPer / 64;      // chunks of a block, and of a lane's
    typedef typename Chunk<T>::vec vec;
    const T* row;
    int vocab, shift;        // shift: entries of the first chunk that come before the row
    int low, high;           // the whole chunks: low .. high
    __device__ __forceinline__ Line(const T* r, int n) : row(r), vocab(n) {
        shift = (int)((uintptr_t)r & 15u) / (int)sizeof(T);
        low = shift > 0 ? 1 : 0;
        high = (vocab + shift) / E - 1;
    }
    __device__ __forceinline__ int blocks() const { return (vocab + shift + kPer * E - 1) / (kPer * E); }
    __device__ __forceinline__ int first(int chunk) const { return chunk * E - shift; }
    __device__ __forceinline__ int block_of(int entry) const { return (entry + shift) / (kPer * E); }
    // the lane's chunk k of block b
    static __device__ __forceinline__ int chunk(int b, int k, int lane) { return b * kPer + k * 64 + lane; }
    // The lane's chunks of block b.  A chunk that is not whole in the row is asked for as the nearest whole one, and mended below: no
    // branch stands around the loads.
    __device__ __forceinline__ void fetch(int b, int lane, vec (&v)[kLoads]) const {
        if (high < low) return;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int i = min(max(chunk(b, k, lane), low), high);
            v[k] = *(const vec*)(row + first(i));
        }
    }
    __device__ __forceinline__ void mend(int b, int lane, vec (&v)[kLoads]) const {
        if (b * kPer >= low && (b + 1) * kPer - 1 <= high) return;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int i = chunk(b, k, lane);
            if (i >= low && i <= high) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int j = first(i) + e;
                v[k][e] = j >= 0 && j < vocab ? row[j] : (T)-INFINITY;
            }
        }
    }
    // chunk i of another row of as many entries, which may begin anywhere
    __device__ __forceinline__ vec beside(const T* other, int i) const {
        vec v;
        const int j0 = first(i);
        if (i >= low && i <= high) return *(const typename Chunk<T>::any*)(other + j0);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] = j0 + e >= 0 && j0 + e < vocab ? other[j0 + e] : (T)-INFINITY;
        return v;
    }
};

// Sums of blocks b = first, first + step, ... < end of a row, by one wave, with a block on its way besides the one at hand.  (A multiply-add in place of the
// difference and the product, and maxima in a third of the instructions, left all times as they were; three blocks on their way made
// 256 requests of 5 drafts 112 us for 94.)
template <typename T>
__device__ __forceinline__ void sum_blocks(const Line<T>& line, float c, int first, int end, int step, BlockSum* out) {
    constexpr int E = Line<T>::E, kLoads = Line<T>::kLoads;
    typedef typename Line<T>::vec vec;
    const int lane = threadIdx.x & 63;
    if (first >= end) return;
    float ref = -INFINITY, at = 0.0f;                // at: what differences are taken from (anchor(ref))
    vec next[kLoads];
    line.fetch(first, lane, next);
    for (int b = first; b < end; b += step) {
        vec v[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) v[k] = next[k];
        if (b + step < end) line.fetch(b + step, lane, next);
        line.mend(b, lane, v);
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            float z[E];
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = (float)v[k][e];
            float top = z[0];
#pragma unroll
            for (int e = 1; e < E; ++e) top = fmaxf(top, z[e]);
            if (__any(top > ref)) {                  // (seldom, after the first)
                const float higher = fmaxf(ref, wave_max_f(top));
                sum *= exp2_hw(fmaxf((ref - higher) * c, -1000.0f));
                ref = higher;
                at = anchor(ref);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) z[e] = share(z[e], at, c);
#pragma unroll
            for (int w = 1; w < E; w *= 2)
#pragma unroll
                for (int e = 0; e + w < E; e += 2 * w) z[e] += z[e + w];
            sum += z[0];
        }
        sum = wave_sum_f(sum);
        if (lane == 0) out[b] = {ref, sum};
    }
}

// what a block's sum counts at the row's largest reference (the factor's second part only where the first has told that it counts: a mask at the type's
// lowest value times it may be past the end, to the other side)
__device__ __forceinline__ float weight_of(float ref, float top, Factor c) {
    const float d = ref - top;
    return d * c.c > -1000.0f ? exp2_hw(c(d)) : 0.0f;
}

// Largest reference and whole sum of a row, by one wave; every lane gets both.
struct Whole {
    float top;
    double sum;
};
__device__ __forceinline__ Whole wave_whole(const BlockSum* table, int blocks, Factor c) {
    const int lane = threadIdx.x & 63;
    const BlockSum none = {-INFINITY, 0.0f}, a = lane < blocks ? table[lane] : none, b = lane + 64 < blocks ? table[lane + 64] : none;
    float top = fmaxf(a.ref, b.ref);
    for (int i = lane + 128; i < blocks; i += 64) top = fmaxf(top, table[i].ref);
    top = wave_max_f(top);
    double sum = (double)a.sum * (double)weight_of(a.ref, top, c) + (double)b.sum * (double)weight_of(b.ref, top, c);
    for (int i = lane + 128; i < blocks; i += 64) sum += (double)table[i].sum * (double)weight_of(table[i].ref, top, c);
    return {top, wave_sum(sum)};
}
__device__ __forceinline__ bool has_mass(double sum) { return sum > 0.0 && sum < INFINITY; }

// Running sum over the lanes (the lane's own in it): lane permutations within rows of 16, then the last lane of a row, and of half a wave, to
// those behind it.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double v) {
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xf, false);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xf, false);
    return v + __hiloint2double(hi, lo);
}
__device__ __forceinline__ double wave_running(double v) {
    v = dpp_add<0x111, 0xf>(v);          // row_shr by 1, 2, 4, 8
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);          // row_bcast 15 to rows 1 and 3
    return dpp_add<0x143, 0xc>(v);       // row_bcast 31 to rows 2 and 3
}
__device__ __forceinline__ int last_lane(unsigned long long mask) { return 63 - __clzll(mask); }
__device__ __forceinline__ double from_lane(double v, int lane) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}

// The lane whose part holds the goal: the first with a part of its own whose running sum passes it; rounding can leave none, then it is the last with
// a part.  -1: none has one.
__device__ __forceinline__ int holder(double own, double running, double goal) {
    const unsigned long long some = __ballot(own > 0.0), passed = __ballot(own > 0.0 && running > goal);
    return passed ? __ffsll((long long)passed) - 1 : (some ? last_lane(some) : -1);
}

// The block, of `blocks` with the sums at(b) >= 0, in which the running sum passes u of the whole, and how much of it is left there.  By one wave.
struct Place {
    int block;               // -1: no block has a share
    double left, total;
};
template <int FEW, typename At>          // FEW: sums of a lane that are asked for at once, and once, if there are no more: each may be a trip to memory
__device__ __forceinline__ Place find_block(int blocks, double u, At at) {
    const int lane = threadIdx.x & 63, each = (blocks + 63) / 64, from = min(lane * each, blocks), to = min(from + each, blocks);
    double own = 0.0, few[FEW];
    if (each <= FEW) {
#pragma unroll
        for (int k = 0; k < FEW; ++k) few[k] = from + k < to ? at(from + k) : 0.0;
#pragma unroll
        for (int k = 0; k < FEW; ++k) own += few[k];
    } else {
        for (int b = from; b < to; ++b) own += at(b);
    }
    const double running = wave_running(own), total = from_lane(running, 63), goal = u * total;
    const int who = holder(own, running, goal);
    double sum = running - own, left = goal - sum;
    int found = from;
    if (each <= FEW) {
        bool done = false;
#pragma unroll
        for (int k = 0; k < FEW; ++k)
            if (few[k] > 0.0 && !done) {
                found = from + k;
                left = goal - sum;
                sum += few[k];
                done = sum > goal;
            }
    } else {
        for (int b = from; b < to; ++b) {
            const double v = at(b);
            if (!(v > 0.0)) continue;
            found = b;
            left = goal - sum;
            sum += v;
            if (sum > goal) break;
        }
    }
    if (who < 0) return {-1, 0.0, total};
    return {__builtin_amdgcn_readlane(found, who), fmax(from_lane(left, who), 0.0), total};
}

// The entry of a block whose running sum passes `left`: its number, -1 if none has a share.  values(k, v): the E values of the lane's chunk k, 64 lanes
// beside each other.  First the chunks' sums over the wave, then the one chunk lane by lane and entry by entry: a lane holds E values and not all.
template <int LOADS, int E, typename Values>
__device__ __forceinline__ int find_entry(double left, Values values) {
    double own[LOADS];
    float v[E];
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
        values(k, v);
        own[k] = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) own[k] += (double)v[e];
    }
    int chunk = -1, last = -1;
    double sum = 0.0, before = 0.0, before_last = 0.0, mine = 0.0, mine_last = 0.0;
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
        const double all = wave_sum(own[k]);
        if (all > 0.0) {
            last = k;
            before_last = sum;
            mine_last = own[k];
            if (chunk < 0 && sum + all > left) {
                chunk = k;
                before = sum;
                mine = own[k];
            }
            sum += all;
        }
    }
    if (last < 0) return -1;
    if (chunk < 0) {                     // (rounding can leave none that is passed)
        chunk = last;
        before = before_last;
        mine = mine_last;
    }
    const double goal = left - before, running = wave_running(mine);
    const int who = holder(mine, running, goal);
#pragma unroll
    for (int k = 0; k < LOADS; ++k)
        if (k == chunk) values(k, v);
    // (every lane looks among its own, the one in question tells)
    double at = running - mine;
    int found = 0;
    bool done = false;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (v[e] > 0.0f && !done) {
            found = e;
            at += (double)v[e];
            done = at > goal;
        }
    return (chunk * 64 + who) * E + __builtin_amdgcn_readlane(found, who);
}

// u in [0, 1)
__device__ __forceinline__ double number(float u) { return (double)fminf(fmaxf(u, 0.0f), 0x1.fffffep-1f); }

// ---- drawing from p ----------------------------------------------------------------------------------------------------------

struct Drawn {
    int token;
    float logp;
};

// Entry of p, without entry `skip` (-1: none is left out) where anything else has a share.  w: of the whole row.  By one wave.
template <typename T>
__device__ __forceinline__ Drawn draw_from(const T* row, int vocab, Factor c, double s, const BlockSum* table, const Whole& w, int skip, float u) {
    typedef Line<T> L;
    const L line(row, vocab);
    const int lane = threadIdx.x & 63, blocks = line.blocks();
    if (!has_mass(w.sum) || u != u) return {-1, NAN};
    typename L::vec raw[L::kLoads];
    auto open = [&](int b) {
        line.fetch(b, lane, raw);
        line.mend(b, lane, raw);
    };
    auto values = [&](int b, float ref, int k, float (&v)[L::E]) {
        const int at = line.first(L::chunk(b, k, lane));
#pragma unroll
        for (int e = 0; e < L::E; ++e) v[e] = at + e == skip ? 0.0f : share((float)raw[k][e], anchor(ref), c.c);
    };
    float skipped = 0.0f;                // the sum of the block that is short of an entry
    const int short_block = skip >= 0 ? line.block_of(skip) : -1;
    if (skip >= 0) {
        open(short_block);
        float v[L::E];
#pragma unroll
        for (int k = 0; k < L::kLoads; ++k) {
            values(short_block, table[short_block].ref, k, v);
#pragma unroll
            for (int e = 0; e < L::E; ++e) skipped += v[e];
        }
        skipped = wave_sum_f(skipped);
    }
    Place p = find_block<1>(blocks, number(u), [&](int b) { return (double)(b == short_block ? skipped : table[b].sum) * (double)weight_of(table[b].ref, w.top, c); });
    if (p.block < 0) {                   // (nothing else has a share: with the entry that was to be left out)
        skip = -1;
        p = find_block<1>(blocks, number(u), [&](int b) { return (double)table[b].sum * (double)weight_of(table[b].ref, w.top, c); });
    }
    const float ref = table[p.block].ref;
    open(p.block);
    const int found = find_entry<L::kLoads, L::E>(p.left / (double)weight_of(ref, w.top, c), [&](int k, float (&v)[L::E]) { values(p.block, ref, k, v); });
    if (found < 0) return {-1, NAN};
    const int token = line.first(p.block * L::kPer) + found;
    return {token, (float)(((double)(float)row[token] - (double)w.top) * s - log_d(w.sum))};
}

// One workgroup a row, its blocks' sums in LDS.  8192 x 131072 bf16 355 us, 6.05 TB/s: memory, with 9 instructions an entry, one of them an exponential,
// close behind; 1001 x 50021 f16 21.7; 8 x 32768 6.2, the launch, the row, the one block again and the token's logit one behind the other.
template <typename T>
__global__ __launch_bounds__(1024) void k_draw_rows(DrawArgs a, int64_t first) {
    extern __shared__ BlockSum sums[];
    const int64_t r = first + blockIdx.x;
    const T* row = (const T*)a.z + r * a.ld;
    const Line<T> line(row, a.vocab);
    sum_blocks<T>(line, a.c.c, (int)(threadIdx.x >> 6), line.blocks(), (int)(blockDim.x >> 6), sums);
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const Drawn d = draw_from<T>(row, a.vocab, a.c, a.s, sums, wave_whole(sums, line.blocks(), a.c), -1, a.uniform[r]);
    if (threadIdx.x == 0) {
        a.tokens[r] = d.token;
        a.logp[r] = d.logp;
    }
}

// Few long rows: their blocks over many workgroups, then a wave a row.
template <typename T>
__global__ __launch_bounds__(kDrawBlock) void k_block_sums(DrawArgs a, int pieces, int64_t most, BlockSum* table) {
    const int64_t r = blockIdx.x / (unsigned)pieces;
    const Line<T> line((const T*)a.z + r * a.ld, a.vocab);
    const int piece = blockIdx.x % (unsigned)pieces, blocks = line.blocks(), each = (blocks + pieces - 1) / pieces;
    sum_blocks<T>(line, a.c.c, piece * each + (int)(threadIdx.x >> 6), min((piece + 1) * each, blocks), kDrawWaves, table + r * most);
}
template <typename T>
__global__ __launch_bounds__(64) void k_draw(DrawArgs a, int64_t most, const BlockSum* table) {
    const int64_t r = blockIdx.x;
    const T* row = (const T*)a.z + r * a.ld;
    table += r * most;
    const Drawn d = draw_from<T>(row, a.vocab, a.c, a.s, table, wave_whole(table, Line<T>(row, a.vocab).blocks(), a.c), -1, a.uniform[r]);
    if (threadIdx.x == 0) {
        a.tokens[r] = d.token;
        a.logp[r] = d.logp;
    }
}

// ---- verification ------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ int length_of(const VerifyArgs& a, int64_t i) {
    if (!a.lengths) return a.drafts;
    const int64_t n = a.lengths[i];
    return n < 0 ? -1 : (n < a.drafts ? (int)n : a.drafts);
}
template <typename T>
__device__ __forceinline__ const T* row_of(const RowSet& s, int64_t i, int t) {
    return (const T*)s.z + i * s.ld_request + (int64_t)t * s.ld;
}

// What is known of a position before its rows are summed, asked for early: two trips to memory, one behind the other.
template <typename T>
__device__ __forceinline__ Asked ask(const VerifyArgs& a, int64_t i, int t, const T* row, const T* drow) {
    const int64_t at = i * a.drafts + t, drafted = a.drafted[at];
    Asked k;
    k.u = a.uniform[at];
    k.given = a.draft_logp ? a.draft_logp[at] : 0.0f;
    k.inside = drafted >= 0 && drafted < a.vocab;
    k.x = k.inside ? (int)drafted : 0;
    k.z = (float)row[k.x];
    k.zq = a.draft.z ? (float)drow[k.x] : 0.0f;
    return k;
}
// Whether a position's token is accepted, and what is drawn from otherwise.  w: of the drafter's row, where it is summed.
__device__ __forceinline__ Position judged(const VerifyArgs& a, const Asked& k, const Whole& p, const Whole& w) {
    Position v = {p.sum, p.top, {}, 0.0f, {}, 0, kFromTarget, 0, 0.0f};
    if (!k.inside || !has_mass(p.sum)) return v;
    double log_q = 0.0;
    if (a.draft.z && !a.draft_logp) {
        if (!has_mass(w.sum)) return v;
        const double log_sum = log_d(w.sum);
        log_q = ((double)k.zq - (double)w.top) * a.draft_s - log_sum;
        v.q_ref = w.top;
        v.q = exponent_of(-log_sum);
    } else if (a.draft.z) {
        log_q = (double)k.given;
        if (!(has_mass(exp(log_q)) && fabsf(k.zq) < INFINITY)) return v;
        v.q_ref = k.zq;
        v.q = exponent_of(log_q);
    }
    const double log_sum = log_d(p.sum), lp = ((double)k.z - (double)p.top) * a.s - log_sum, q = exp(log_q);
    v.p = exponent_of(-log_sum);
    v.mode = a.draft.z ? kRest : kWithout;
    v.x = k.x;
    v.accepted = q > 0.0 && (double)(k.u < 0.0f ? 0.0f : k.u) * q < exp(lp);
    v.logp = (float)lp;
    return v;
}
__device__ __forceinline__ Position behind_last(const Whole& p) { return {p.sum, p.top, {}, 0.0f, {}, 0, kFromTarget, 0, 0.0f}; }

// -1 and 0 from position `from` of a request on, by `threads` threads
__device__ __forceinline__ void blanks(const VerifyArgs& a, int64_t i, int from, int thread, int threads) {
    const int64_t out = i * (a.drafts + 1);
    for (int t = from + thread; t <= a.drafts; t += threads) {
        a.tokens[out + t] = -1;
        a.logp[out + t] = 0.0f;
    }
}

// max(p - q, 0) of a chunk.  (A difference that is no number, or without end, makes one that is none, and p is drawn from instead.)
template <typename T>
__device__ __forceinline__ void rest_of(const VerifyArgs& a, const Position& d, typename Line<T>::vec p, typename Line<T>::vec q, float (&v)[Line<T>::E]) {
#pragma unroll
    for (int e = 0; e < Line<T>::E; ++e) {
        const float r = mass((float)p[e], d.top, a.c, d.p) - mass((float)q[e], d.q_ref, a.draft_c, d.q);
        v[e] = r > 0.0f ? r : r * 0.0f;
    }
}

// The last token of a request, at position t, by one wave.  rest(k): the sum of max(p - q, 0) over 64 chunks from 64 k on, where that is drawn from.
template <typename T, typename At>
__device__ __forceinline__ void finish(const VerifyArgs& a, int64_t i, int t, const Position& d, const BlockSum* table, At rest) {
    typedef Line<T> L;
    const T* row = row_of<T>(a.target, i, t);
    const float v = a.last_uniform[i];
    Drawn got = {-1, NAN};
    bool found = false;
    if (d.mode == kRest && v == v) {
        const L line(row, a.vocab);
        const Place p = find_block<8>(line.blocks() * L::kLoads, number(v), rest);
        if (p.block >= 0 && has_mass(p.total)) {         // (a sum that is no number makes the total one)
            const int chunk = p.block * 64 + (int)(threadIdx.x & 63);
            const typename L::vec z = line.beside(row, chunk), zq = line.beside(row_of<T>(a.draft, i, t), chunk);
            const int e = find_entry<1, L::E>(p.left, [&](int, float (&out)[L::E]) { rest_of<T>(a, d, z, zq, out); });
            found = e >= 0;
            if (found) {
                got.token = line.first(p.block * 64) + e;
                got.logp = (float)(((double)(float)row[got.token] - (double)d.top) * a.s - log_d(d.sum));
            }
        }
    }
    if (!found) got = draw_from<T>(row, a.vocab, a.c, a.s, table, {d.top, d.sum}, d.mode == kWithout ? d.x : -1, v);
    if ((threadIdx.x & 63) == 0) {
        const int64_t out = i * (a.drafts + 1) + t;
        a.tokens[out] = got.token;
        a.logp[out] = got.logp;
        a.count[i] = t + (got.token >= 0 ? 1 : 0);
    }
}

// Sums of max(p - q, 0) over 64 chunks each, number first, first + step, ... < end, by one wave, two of them at once: put(number, sum).  (Finer than the
// blocks: the work spreads, and the one wave that finds the token has 64 chunks to go through.)
constexpr int kRestAtOnce = 2;
template <typename T, typename Put>
__device__ __forceinline__ void sum_rest(const VerifyArgs& a, const Position& d, const Line<T>& line, const T* drow, int first, int end, int step, Put put) {
    typedef Line<T> L;
    const int lane = threadIdx.x & 63;
    for (int n = first; n < end; n += kRestAtOnce * step) {
        typename L::vec p[kRestAtOnce], q[kRestAtOnce];
#pragma unroll
        for (int k = 0; k < kRestAtOnce; ++k) {
            p[k] = line.beside(line.row, (n + k * step) * 64 + lane);
            q[k] = line.beside(drow, (n + k * step) * 64 + lane);
        }
#pragma unroll
        for (int k = 0; k < kRestAtOnce; ++k) {
            float v[L::E], sum = 0.0f;
            rest_of<T>(a, d, p[k], q[k], v);
#pragma unroll
            for (int e = 0; e < L::E; ++e) sum += v[e];
            const double all = wave_sum((double)sum);
            if (lane == 0 && n + k * step < end) put(n + k * step, all);
        }
    }
}

// A workgroup a request, position by position, up to the first token that is not accepted: no row behind it is read.  256 requests of 5 drafts x 131072 f16 93 us for
// 357 MB: 9 to 10 us a row of 256 kB, as fast as one compute unit reads and adds, seven rows where the chain is longest.
template <typename T>
__global__ __launch_bounds__(1024) void k_verify_requests(VerifyArgs a, int64_t first, int64_t most) {
    extern __shared__ BlockSum sums[];                  // of the target's row, then of the drafter's, or of the chunks of max(p - q, 0)
    __shared__ Position at;
    const int64_t i = first + blockIdx.x, out = i * (a.drafts + 1);
    const int n = length_of(a, i), wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if (n < 0) {
        blanks(a, i, 0, threadIdx.x, blockDim.x);
        if (threadIdx.x == 0) a.count[i] = 0;
        return;
    }
    int t = 0;
    for (;; ++t) {
        const T *row = row_of<T>(a.target, i, t), *drow = a.draft.z && t < n ? row_of<T>(a.draft, i, t) : row;
        const Line<T> line(row, a.vocab), dline(drow, a.vocab);
        Asked asked = {};
        if (t < n) asked = ask<T>(a, i, t, row, drow);
        const bool both = a.draft.z && !a.draft_logp && t < n;
        const int half = both && waves > 1 ? (waves + 1) / 2 : waves;
        if (wave < half) sum_blocks<T>(line, a.c.c, wave, line.blocks(), half, sums);
        if (both && (wave >= half || waves == 1)) sum_blocks<T>(dline, a.draft_c.c, waves == 1 ? 0 : wave - half, dline.blocks(), waves == 1 ? 1 : waves - half, sums + most);
        __syncthreads();
        if (wave == 0) {
            const Whole p = wave_whole(sums, line.blocks(), a.c);
            const Position v = t < n ? judged(a, asked, p, both ? wave_whole(sums + most, dline.blocks(), a.draft_c) : Whole{0.0f, 0.0}) : behind_last(p);
            if (threadIdx.x == 0) {
                at = v;
                if (v.accepted) {
                    a.tokens[out + t] = asked.x;
                    a.logp[out + t] = v.logp;
                }
            }
        }
        __syncthreads();
        if (!at.accepted) break;                        // (at position n it is not)
    }
    blanks(a, i, t + 1, threadIdx.x, blockDim.x);
    const Position d = at;
    double* rest = (double*)(sums + most);
    if (d.mode == kRest) {
        const Line<T> line(row_of<T>(a.target, i, t), a.vocab);
        const T* drow = row_of<T>(a.draft, i, t);
        sum_rest<T>(a, d, line, drow, wave, line.blocks() * Line<T>::kLoads, waves, [&](int k, double s) { rest[k] = s; });
        __syncthreads();
    }
    if (wave == 0) finish<T>(a, i, t, d, sums, [&](int k) { return rest[k]; });
}

// Few requests: their rows' blocks over many workgroups.  The target's rows up to a request's length, and (rows behind those) the drafter's before
// it.  For the next launch what has to be asked for is there in one piece, and the requests' tickets are cleared.
template <typename T>
__global__ __launch_bounds__(kDrawBlock) void k_verify_sums(VerifyArgs a, int64_t first, int pieces, int64_t most, BlockSum* target, BlockSum* draft,
                                                            Asked* asked, unsigned* tickets) {
    int64_t r = first + blockIdx.x / (unsigned)pieces;
    const int piece = blockIdx.x % (unsigned)pieces;
    if (piece == 0 && r < a.requests && threadIdx.x == 0) tickets[r] = 0;
    const int64_t of_target = a.requests * a.target.each;
    const bool drafter = r >= of_target;
    if (drafter) r -= of_target;
    const RowSet& set = drafter ? a.draft : a.target;
    const int64_t i = r / set.each;
    const int t = (int)(r - i * set.each), n = length_of(a, i);
    if (n < 0 || t > n - (drafter ? 1 : 0)) return;
    const T* row = row_of<T>(set, i, t);
    const Line<T> line(row, a.vocab);
    const int blocks = line.blocks(), each = (blocks + pieces - 1) / pieces;
    if (piece == 0 && !drafter && t < n && threadIdx.x == 0) asked[i * a.drafts + t] = ask<T>(a, i, t, row, a.draft.z ? row_of<T>(a.draft, i, t) : row);
    sum_blocks<T>(line, drafter ? a.draft_c.c : a.c.c, piece * each + (int)(threadIdx.x >> 6), min((piece + 1) * each, blocks), kDrawWaves,
                  (drafter ? draft : target) + r * most);
}

// The first token of a request that is not accepted, the sums of max(p - q, 0) there, and its last token.  Every workgroup finds out the first
// for itself, and the last to be done the third (the sums are read in their own order, whichever that is): a launch each less.  32 requests of 4
// drafts x 131072 bf16 12 us behind 11 for the sums (42 MB): trips to memory one behind the other, not bytes (11 MB).
constexpr int kRestWaves = 8;            // of a workgroup: as many positions are judged at once
template <typename T>
__global__ __launch_bounds__(kRestWaves * 64) void k_verify_rest(VerifyArgs a, int64_t first, int pieces, int64_t most, const BlockSum* target,
                                                                 const BlockSum* draft, const Asked* asked, double* rest, unsigned* tickets) {
    __shared__ Position found[kRestWaves];
    __shared__ int last;
    const int64_t i = first + blockIdx.x / (unsigned)pieces, out = i * (a.drafts + 1);
    const int piece = blockIdx.x % (unsigned)pieces, n = length_of(a, i), wave = threadIdx.x >> 6;
    if (n < 0) {
        if (piece == 0) blanks(a, i, 0, threadIdx.x, blockDim.x);
        if (piece == 0 && threadIdx.x == 0) a.count[i] = 0;
        return;
    }
    const BlockSum* table = target + i * a.target.each * most;
    int t = 0;
    Position d;
    for (bool more = true; more;) {
        const int mine = t + wave, some = min(kRestWaves, n + 1 - t);
        if (wave < some) {
            const T* row = row_of<T>(a.target, i, mine);
            const int blocks = Line<T>(row, a.vocab).blocks();
            if (mine < n) {
                const T* drow = a.draft.z ? row_of<T>(a.draft, i, mine) : row;
                const Asked known = asked[i * a.drafts + mine];
                const Whole p = wave_whole(table + mine * most, blocks, a.c);
                const Position v = judged(a, known, p, a.draft.z && !a.draft_logp ? wave_whole(draft + (i * a.draft.each + mine) * most, Line<T>(drow, a.vocab).blocks(), a.draft_c)
                                                                                     : Whole{0.0f, 0.0});
                if ((threadIdx.x & 63) == 0) found[wave] = v;
            } else {
                const Whole p = wave_whole(table + mine * most, blocks, a.c);
                if ((threadIdx.x & 63) == 0) found[wave] = behind_last(p);
            }
        }
        __syncthreads();
        int w = 0;
        while (w < some && found[w].accepted) ++w;
        if (piece == 0 && (int)threadIdx.x < w) {
            a.tokens[out + t + threadIdx.x] = found[threadIdx.x].x;
            a.logp[out + t + threadIdx.x] = found[threadIdx.x].logp;
        }
        t += w;
        more = w == some;                               // (at position n none is accepted)
        if (!more) d = found[w];
        __syncthreads();
    }
    if (piece == 0) blanks(a, i, t + 1, threadIdx.x, blockDim.x);
    table += t * most;
    if (d.mode != kRest) {
        if (piece == 0 && wave == 0) finish<T>(a, i, t, d, table, [](int) { return 0.0; });
        return;
    }
    double* sums = rest + i * most * Line<T>::kLoads;
    const Line<T> line(row_of<T>(a.target, i, t), a.vocab);
    const T* drow = row_of<T>(a.draft, i, t);
    const int all = line.blocks() * Line<T>::kLoads, each = (all + pieces - 1) / pieces;
    sum_rest<T>(a, d, line, drow, piece * each + wave, min((piece + 1) * each, all), kRestWaves, [&](int k, double s) { publish(&sums[k], s); });
    if (!arrive_is_last(&tickets[i], &last, (unsigned)pieces)) return;
    if (wave == 0) finish<T>(a, i, t, d, table, [&](int k) { return observe(&sums[k]); });
}

constexpr int64_t kThreadsMax = (1ll << 32) - 1;      // of a launch: longer batches take several

// Pieces of each of `rows` rows: enough workgroups to fill the card, as far as each of their waves has a block.
int pieces_of(int64_t rows, int64_t blocks, int waves, int64_t workgroups) {
    const int64_t want = (workgroups + rows - 1) / rows, most = (blocks + waves - 1) / waves;
    return (int)(want < most ? want : most);
}

// f(first, count): `each` workgroups of so many threads for each of the rows first .. first + count - 1
template <typename F>
hipError_t in_launches(int64_t rows, int64_t each, int64_t threads, F f) {
    const int64_t most = kThreadsMax / (each * threads);
    for (int64_t r = 0; r < rows; r += most) {
        f(r, rows - r < most ? rows - r : most);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Waves that take a row together; 0: it is split over workgroups.  us of calls in a row, split / 4 / 8 / 16 waves: 8192 x 131072 bf16 398 / 363 / 358 / 381,
// 1001 x 50021 f16 27.6 / 22.8 / 23.6 / 30.6, 300 x 131072 f32 37.1 / 42.5 / 35.8 / 39.1, 100 x 131072 bf16 12.2 / 15.5 / 13.8 / 12.8, 40 x 100000 f32 11.1 /
// 23.0 / 15.1 / 13.4, 1 x 65536 bf16 10.4 / 9.4 / 8.3 / 7.8, 8 x 32768 9.5 / 7.2 / 6.7 / 6.5, 8192 x 4000 30 / 29 / 42 / 59.
int row_waves(int64_t rows, int64_t blocks) {
    if (rows <= 128 && blocks > 56) return 0;
    const int64_t want = rows <= 256 ? 16 : (blocks >= 32 ? 8 : 4);
    return (int)(want < blocks ? want : blocks);
}

// Whether a request's positions are taken one after another by one workgroup, which then reads no row in vain but goes no faster than its
// compute unit.  us, so / by many workgroups, log-probabilities given where not said:
//                                  128          144          160          192          256 requests
// 4 drafts x 131072 bf16           72 / 60      72 / 64      74 / 67      75 / 78      77 / 95
// the same, both sides summed      103 / 88     104 / 96     104 / 104    106 / 118    113 / 148
// 5 x 131072 f16                   85 / 68      85 / 74      86 / 79      87 / 94      90 / 111
// 3 x 50021 f32                    42 / 40      41 / 43      42 / 46      44 / 54      47 / 66
// 2 x 32768 f16                    19.8 / 19.9  20.3 / 21.0  20.4 / 22.9  21.0 / 25.4  22.7 / 30.1
// 2 of 3 x 32768 12.4 / 11.3.  They meet between 128 and 190, whatever the drafts and entries are; from 160 on neither is more than a tenth behind where it is taken.
bool by_request(int64_t requests) { return requests >= 160; }

template <typename T>
hipError_t draw_rows(const DrawArgs& a, void* ws, hipStream_t st) {
    const int64_t most = blocks_of(a.vocab, sizeof(T));
    const int waves = row_waves(a.rows, most);
    if (waves)
        return in_launches(a.rows, 1, waves * 64, [&](int64_t first, int64_t n) {
            hipLaunchKernelGGL(k_draw_rows<T>, dim3((unsigned)n), dim3(waves * 64), most * sizeof(BlockSum), st, a, first);
        });
    const int pieces = pieces_of(a.rows, most, kDrawWaves, 2048);
    BlockSum* table = (BlockSum*)ws;
    hipLaunchKernelGGL(k_block_sums<T>, dim3((unsigned)(a.rows * pieces)), dim3(kDrawBlock), 0, st, a, pieces, most, table);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_draw<T>, dim3((unsigned)a.rows), dim3(64), 0, st, a, most, (const BlockSum*)table);
    return hipGetLastError();
}

template <typename T>
hipError_t verify_rows(const VerifyArgs& a, void* ws, hipStream_t st) {
    const int64_t most = blocks_of(a.vocab, sizeof(T)), n = a.requests;
    const bool both = a.draft.z && !a.draft_logp;
    if (by_request(n)) {
        const int64_t want = most * (both ? 2 : 1), waves = want < 16 ? want : 16;      // (of 4 kB each: a compute unit's share of the card)
        return in_launches(n, 1, waves * 64, [&](int64_t first, int64_t c) {
            hipLaunchKernelGGL(k_verify_requests<T>, dim3((unsigned)c), dim3((unsigned)waves * 64), most * (a.draft.z ? 1 + kBlockBytes / 1024 : 1) * sizeof(BlockSum), st, a, first, most);
        });
    }
    const VerifySpace sp = verify_space(n, a.drafts, a.vocab, sizeof(T), a.draft.z, both);
    char* at = (char*)ws;
    BlockSum *target = (BlockSum*)at, *draft = (BlockSum*)(at + sp.draft);
    double* rest = (double*)(at + sp.rest);
    Asked* asked = (Asked*)(at + sp.asked);
    unsigned* tickets = (unsigned*)(at + sp.tickets);
    const int64_t rows = n * a.target.each + (both ? n * a.draft.each : 0);
    int pieces = pieces_of(rows, most, kDrawWaves, 4096);
    hipError_t e = in_launches(rows, pieces, kDrawBlock, [&](int64_t first, int64_t c) {
        hipLaunchKernelGGL(k_verify_sums<T>, dim3((unsigned)(c * pieces)), dim3(kDrawBlock), 0, st, a, first, pieces, most, target, draft, asked, tickets);
    });
    if (e != hipSuccess) return e;
    pieces = a.draft.z ? pieces_of(n, most * Line<T>::kLoads / kRestAtOnce, kRestWaves, 2048) : 1;
    return in_launches(n, pieces, kRestWaves * 64, [&](int64_t first, int64_t c) {
        hipLaunchKernelGGL(k_verify_rest<T>, dim3((unsigned)(c * pieces)), dim3(kRestWaves * 64), 0, st, a, first, pieces, most, (const BlockSum*)target,
                           (const BlockSum*)draft, (const Asked*)asked, rest, tickets);
    });
}

template <typename F>
hipError_t by_type(int dtype, F f) {
    return dtype == LBFGSB_F32 ? f(float{}) : (dtype == LBFGSB_BF16 ? f(__bf16{}) : f(_Float16{}));
}

size_t rounded(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

size_t draw_space(int64_t rows, int64_t vocab, int size) {
    const int64_t blocks = blocks_of(vocab, size);
    return rows == 0 || row_waves(rows, blocks) ? 0 : rounded((size_t)(rows * blocks) * sizeof(BlockSum));
}

VerifySpace verify_space(int64_t requests, int64_t drafts, int64_t vocab, int size, bool drafter, bool both) {
    const size_t most = (size_t)blocks_of(vocab, size), n = (size_t)requests;
    if (n == 0 || by_request(requests)) return {0, 0, 0, 0, 0};
    VerifySpace s;
    s.draft = rounded(n * (drafts + 1) * most * sizeof(BlockSum));
    s.rest = s.draft + (both ? rounded(n * drafts * most * sizeof(BlockSum)) : 0);
    s.asked = s.rest + (drafter ? rounded(n * most * (kBlockBytes / 1024) * sizeof(double)) : 0);
    s.tickets = s.asked + rounded(n * drafts * sizeof(Asked));
    s.whole = s.tickets + rounded(n * sizeof(unsigned));
    return s;
}

hipError_t launch_draw(const DrawArgs& a, int dtype, void* ws, hipStream_t st) {
    if (a.rows == 0) return hipSuccess;
    return by_type(dtype, [&](auto e) { return draw_rows<decltype(e)>(a, ws, st); });
}

hipError_t launch_verify(const VerifyArgs& a, int dtype, void* ws, hipStream_t st) {
    if (a.requests == 0) return hipSuccess;
    return by_type(dtype, [&](auto e) { return verify_rows<decltype(e)>(a, ws, st); });
}

}  // namespace lb
