// Tokens drawn from rows of logits by given numbers, and drafted tokens verified against the target's rows.
//
// A token is the first entry at which the running sum of p passes u.  With e_j = 2^((z_j - ref) c) a row is read once, in blocks of
// 4 kB whose sums are kept (8 bytes a block: 0.2 % of the row); in 64 bits the blocks' sums tell the block in which u S is
// passed, S being the whole row's, and that block alone is read again, lane by lane and entry by entry.  Sums of a block are in 32 bits and off by
// 2^-24 of the block's own, all else is in 64 bits.
//
// Verification: sums of all the target's rows (and of the drafter's, where its log-probabilities are not at hand) in one launch; the first
// token that is not accepted follows from them; in a second, workgroups sum blocks of max(p - q, 0) at it, and the last of a request's to be done
// finds the token.
#include "draws.h"

namespace lb {

namespace {

constexpr int kDrawBlock = 256, kDrawWaves = kDrawBlock / 64;

// 2^((z - ref) c) as it enters the sums of blocks: c is the factor's first part alone (2^-25 of the distance to the wave's largest so far,
// to one side; joins of blocks take both parts).
__device__ __forceinline__ float share(float z, float ref, float c) { return exp2_hw((z - ref) * c); }
// The same with the factor's second part and the rounding of the exponent put right: for differences p - q, and references that are not the largest.
__device__ __forceinline__ float share_exact(float z, float ref, Factor c) {
    const float d = z - ref, a = d * c.c, e = exp2_hw(a);
    const float rest = a > -1000.0f && a < 1000.0f ? fmaf(d, c.low, fmaf(d, c.c, -a)) : 0.0f;
    return fmaf(e, rest * 0.693147181f, e);
}

// A row as it is read in blocks: chunks of 16 bytes on boundaries of the logits, of which the first and the last may hold less of the row.
template <typename T>
struct Line {
    static constexpr int E = Chunk<T>::E, kPer = kBlockBytes / 16, kLoads = kPer / 64, kEntries = kLoads * E;    // chunks of a block; a lane's
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
    // the lane's chunk k of block b: SPREAD, 64 lanes beside each other; else the lane's four are beside each other
    template <bool SPREAD>
    static __device__ __forceinline__ int chunk(int b, int k, int lane) { return b * kPer + (SPREAD ? k * 64 + lane : lane * kLoads + k); }
    // The lane's chunks of block b.  A chunk that is not whole in the row is asked for as the nearest whole one, and mended below: no
    // branch stands around the loads.
    template <bool SPREAD>
    __device__ __forceinline__ void fetch(int b, int lane, vec (&v)[kLoads]) const {
        if (high < low) return;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int i = min(max(chunk<SPREAD>(b, k, lane), low), high);
            v[k] = *(const vec*)(row + first(i));
        }
    }
    template <bool SPREAD>
    __device__ __forceinline__ void mend(int b, int lane, vec (&v)[kLoads]) const {
        if (b * kPer >= low && (b + 1) * kPer - 1 <= high) return;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int i = chunk<SPREAD>(b, k, lane);
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

// Sums of blocks b = first, first + step, ... < end of a row, by one wave.
template <typename T>
__device__ __forceinline__ void sum_blocks(const Line<T>& line, float c, int first, int end, int step, BlockSum* out) {
    constexpr int E = Line<T>::E, kLoads = Line<T>::kLoads;
    typedef typename Line<T>::vec vec;
    const int lane = threadIdx.x & 63;
    if (first >= end) return;
    float ref = -INFINITY, at = 0.0f;                // at: what differences are taken from (anchor(ref))
    vec next[kLoads];
    line.template fetch<true>(first, lane, next);
    for (int b = first; b < end; b += step) {
        vec v[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) v[k] = next[k];
        if (b + step < end) line.template fetch<true>(b + step, lane, next);
        line.template mend<true>(b, lane, v);
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

// what a block's sum counts at the row's largest reference
__device__ __forceinline__ float weight_of(float ref, float top, Factor c) { return exp2_hw(below(ref, top, c)); }

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
template <typename At>
__device__ __forceinline__ Place find_block(int blocks, double u, At at) {
    const int lane = threadIdx.x & 63, each = (blocks + 63) / 64, from = min(lane * each, blocks), to = min(from + each, blocks);
    double own = 0.0;
    for (int b = from; b < to; ++b) own += at(b);
    const double running = wave_running(own), total = from_lane(running, 63), goal = u * total;
    const int who = holder(own, running, goal);
    double sum = running - own, left = goal - sum;
    int found = from;
    if (each > 1)
        for (int b = from; b < to; ++b) {
            const double v = at(b);
            if (!(v > 0.0)) continue;
            found = b;
            left = goal - sum;
            sum += v;
            if (sum > goal) break;
        }
    if (who < 0) return {-1, 0.0, total};
    return {__builtin_amdgcn_readlane(found, who), fmax(from_lane(left, who), 0.0), total};
}

// The entry, of a wave's N a lane, one lane's behind another's, whose running sum passes `left`: its number, -1 if none has a share.
template <int N>
__device__ __forceinline__ int find_entry(const float (&v)[N], double left) {
    double own = 0.0;
#pragma unroll
    for (int e = 0; e < N; ++e) own += (double)v[e];
    const double running = wave_running(own);
    const int who = holder(own, running, left);
    if (who < 0) return -1;
    // (every lane looks among its own, the one in question tells)
    double sum = running - own;
    int found = 0;
    bool done = false;
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (v[e] > 0.0f && !done) {
            found = e;
            sum += (double)v[e];
            done = sum > left;
        }
    return who * N + __builtin_amdgcn_readlane(found, who);
}

// u in [0, 1)
__device__ __forceinline__ double number(float u) { return (double)fminf(fmaxf(u, 0.0f), 0x1.fffffep-1f); }

// ---- drawing from p ----------------------------------------------------------------------------------------------------------

struct Drawn {
    int token;
    float logp;
};

// Entry of p, without entry `skip` (-1: none is left out) where anything else has a share.  By one wave.
template <typename T>
__device__ __forceinline__ Drawn draw_from(const T* row, int vocab, Factor c, double s, const BlockSum* table, int skip, float u) {
    typedef Line<T> L;
    const L line(row, vocab);
    const int lane = threadIdx.x & 63, blocks = line.blocks();
    auto entries = [&](int b, float ref, int without, float (&v)[L::kEntries]) {
        typename L::vec raw[L::kLoads];
        line.template fetch<false>(b, lane, raw);
        line.template mend<false>(b, lane, raw);
#pragma unroll
        for (int k = 0; k < L::kLoads; ++k)
#pragma unroll
            for (int e = 0; e < L::E; ++e) {
                const bool gone = line.first(L::template chunk<false>(b, k, lane)) + e == without;
                v[k * L::E + e] = gone ? 0.0f : share((float)raw[k][e], anchor(ref), c.c);
            }
    };
    const Whole w = wave_whole(table, blocks, c);
    if (!has_mass(w.sum) || u != u) return {-1, NAN};
    float v[L::kEntries], skipped = 0.0f;      // skipped: the sum of the block that is short of an entry
    const int short_block = skip >= 0 ? line.block_of(skip) : -1;
    if (skip >= 0) {
        entries(short_block, table[short_block].ref, skip, v);
#pragma unroll
        for (int e = 0; e < L::kEntries; ++e) skipped += v[e];
        skipped = wave_sum_f(skipped);
    }
    auto at = [&](int b) { return (double)(b == short_block ? skipped : table[b].sum) * (double)weight_of(table[b].ref, w.top, c); };
    Place p = find_block(blocks, number(u), at);
    if (p.block < 0) {                   // (nothing else has a share: with the entry that was to be left out)
        skip = -1;
        p = find_block(blocks, number(u), [&](int b) { return (double)table[b].sum * (double)weight_of(table[b].ref, w.top, c); });
    }
    const float ref = table[p.block].ref;
    entries(p.block, ref, skip, v);
    const int found = find_entry(v, p.left / (double)weight_of(ref, w.top, c));
    if (found < 0) return {-1, NAN};
    const int token = line.first(p.block * L::kPer) + found;
    return {token, (float)(((double)(float)row[token] - (double)w.top) * s - log_d(w.sum))};
}

// One workgroup a row, its blocks' sums in LDS.
template <typename T>
__global__ __launch_bounds__(1024) void k_draw_rows(DrawArgs a, int64_t first) {
    extern __shared__ BlockSum sums[];
    const int64_t r = first + blockIdx.x;
    const T* row = (const T*)a.z + r * a.ld;
    const Line<T> line(row, a.vocab);
    sum_blocks<T>(line, a.c.c, (int)(threadIdx.x >> 6), line.blocks(), (int)(blockDim.x >> 6), sums);
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const Drawn d = draw_from<T>(row, a.vocab, a.c, a.s, sums, -1, a.uniform[r]);
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
    const Drawn d = draw_from<T>((const T*)a.z + r * a.ld, a.vocab, a.c, a.s, table + r * most, -1, a.uniform[r]);
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

// Sums of the rows that may be asked for: the target's at positions up to a request's length, and (rows behind those) the drafter's before
// it.  The requests' tickets are cleared for the next launch.
template <typename T>
__global__ __launch_bounds__(kDrawBlock) void k_verify_sums(VerifyArgs a, int64_t first, int pieces, int64_t most, BlockSum* target, BlockSum* draft,
                                                            unsigned* tickets) {
    int64_t r = first + blockIdx.x / (unsigned)pieces;
    const int piece = blockIdx.x % (unsigned)pieces;
    if (tickets && piece == 0 && r < a.requests && threadIdx.x == 0) tickets[r] = 0;
    const int64_t of_target = a.requests * a.target.each;
    const bool drafter = r >= of_target;
    if (drafter) r -= of_target;
    const RowSet& set = drafter ? a.draft : a.target;
    const int64_t i = r / set.each;
    const int t = (int)(r - i * set.each), n = length_of(a, i);
    if (n < 0 || t > n - (drafter ? 1 : 0)) return;
    const Line<T> line(row_of<T>(set, i, t), a.vocab);
    const int blocks = line.blocks(), each = (blocks + pieces - 1) / pieces;
    sum_blocks<T>(line, drafter ? a.draft_c.c : a.c.c, piece * each + (int)(threadIdx.x >> 6), min((piece + 1) * each, blocks), kDrawWaves,
                  (drafter ? draft : target) + r * most);
}

// One position, by one wave; every lane gets the result.
struct Verdict {
    int accepted;
    float logp;              // of the drafted token, accepted
    Decision next;           // what is drawn from otherwise
};
template <typename T>
__device__ __forceinline__ Verdict judge(const VerifyArgs& a, int64_t i, int t, int64_t most, const BlockSum* target, const BlockSum* draft) {
    const int64_t at = i * a.drafts + t;
    const int64_t drafted = a.drafted[at];
    const T *row = row_of<T>(a.target, i, t), *drow = a.draft.z ? row_of<T>(a.draft, i, t) : row;
    const bool summed = a.draft.z && !a.draft_logp;
    // (all that is needed is asked for before anything is waited for)
    const int x = drafted >= 0 && drafted < a.vocab ? (int)drafted : 0;
    const float u = a.uniform[at], given = a.draft_logp ? a.draft_logp[at] : 0.0f, z = (float)row[x], zq = (float)drow[x];
    const Whole p = wave_whole(target + (i * a.target.each + t) * most, Line<T>(row, a.vocab).blocks(), a.c);
    Verdict v = {0, 0.0f, {t, kFromTarget, 0, 0.0f, 0.0f, 0.0f, 0.0f}};
    if (x != drafted || !has_mass(p.sum)) return v;
    double q = 1.0;
    if (a.draft.z) {
        if (summed) {
            const Whole w = wave_whole(draft + (i * a.draft.each + t) * most, Line<T>(drow, a.vocab).blocks(), a.draft_c);
            if (!has_mass(w.sum)) return v;
            q = exp(((double)zq - (double)w.top) * a.draft_s) / w.sum;
            v.next.q_ref = w.top;
            v.next.q_factor = (float)(1.0 / w.sum);
        } else {
            q = exp((double)given);
            if (!(has_mass(q) && fabsf(zq) < INFINITY)) return v;
            v.next.q_ref = zq;
            v.next.q_factor = (float)q;
        }
        v.next.mode = kRest;
        v.next.m = p.top;
        v.next.inv = (float)(1.0 / p.sum);
    } else {
        v.next.mode = kWithout;
        v.next.x = x;
    }
    const double lp = ((double)z - (double)p.top) * a.s - log_d(p.sum);
    v.accepted = q > 0.0 && (double)u * q < exp(lp);
    v.logp = (float)lp;
    return v;
}

// Goes through a request's drafted tokens, four at a time.  `tell`: writes what is accepted and the blanks behind it.
template <typename T>
__device__ __forceinline__ Decision decide(const VerifyArgs& a, int64_t i, int64_t most, const BlockSum* target, const BlockSum* draft, bool tell) {
    __shared__ Verdict found[kDrawWaves];
    const int wave = threadIdx.x >> 6, n = length_of(a, i);
    const int64_t out = i * (a.drafts + 1);
    Decision d = {n, kFromTarget, 0, 0.0f, 0.0f, 0.0f, 0.0f};
    int accepted = max(n, 0);
    for (int t0 = 0; t0 < n; t0 += kDrawWaves) {
        const int some = min(kDrawWaves, n - t0);
        if (wave < some) {
            const Verdict v = judge<T>(a, i, t0 + wave, most, target, draft);
            if ((threadIdx.x & 63) == 0) found[wave] = v;
        }
        __syncthreads();
        int w = 0;
        while (w < some && found[w].accepted) ++w;
        if (tell && (int)threadIdx.x < w) {
            const int t = t0 + (int)threadIdx.x;
            a.tokens[out + t] = a.drafted[i * a.drafts + t];
            a.logp[out + t] = found[threadIdx.x].logp;
        }
        if (w < some) {
            d = found[w].next;
            accepted = t0 + w;
            break;
        }
        __syncthreads();
    }
    if (tell)
        for (int t = (n < 0 ? 0 : accepted + 1) + (int)threadIdx.x; t <= a.drafts; t += kDrawBlock) {
            a.tokens[out + t] = -1;
            a.logp[out + t] = 0.0f;
        }
    if (tell && n < 0 && threadIdx.x == 0) a.count[i] = 0;
    return d;
}

// max(p - q, 0) of the lane's entries of block b.  (A difference that is no number stays one, and p is drawn from instead.)
template <typename T, bool SPREAD>
__device__ __forceinline__ void rest_of(const Line<T>& line, const T* drow, int b, const VerifyArgs& a, const Decision& d, float (&v)[Line<T>::kEntries]) {
    typedef Line<T> L;
    const int lane = threadIdx.x & 63;
    typename L::vec p[L::kLoads], q[L::kLoads];
    line.template fetch<SPREAD>(b, lane, p);
#pragma unroll
    for (int k = 0; k < L::kLoads; ++k) q[k] = line.beside(drow, L::template chunk<SPREAD>(b, k, lane));
    line.template mend<SPREAD>(b, lane, p);
#pragma unroll
    for (int k = 0; k < L::kLoads; ++k)
#pragma unroll
        for (int e = 0; e < L::E; ++e) {
            const float r = share_exact((float)p[k][e], d.m, a.c) * d.inv - share_exact((float)q[k][e], d.q_ref, a.draft_c) * d.q_factor;
            v[k * L::E + e] = r <= 0.0f ? 0.0f : r;
        }
}

// The last token of a request, by one wave.  rest: sums of the blocks of max(p - q, 0), where that is drawn from.
template <typename T>
__device__ __forceinline__ void finish(const VerifyArgs& a, int64_t i, const Decision& d, int64_t most, const BlockSum* target, const double* rest) {
    typedef Line<T> L;
    const T* row = row_of<T>(a.target, i, d.t);
    const BlockSum* table = target + (i * a.target.each + d.t) * most;
    const float v = a.last_uniform[i];
    Drawn got = {-1, NAN};
    bool found = false;
    if (d.mode == kRest && v == v) {
        const L line(row, a.vocab);
        const Place p = find_block(line.blocks(), number(v), [&](int b) { return observe(&rest[b]); });
        if (p.block >= 0 && has_mass(p.total)) {         // (a sum that is no number makes the total one)
            found = true;
            float part[L::kEntries];
            rest_of<T, false>(line, row_of<T>(a.draft, i, d.t), p.block, a, d, part);
            const int e = find_entry(part, p.left);
            const Whole w = wave_whole(table, line.blocks(), a.c);
            if (e >= 0) {
                got.token = line.first(p.block * L::kPer) + e;
                got.logp = (float)(((double)(float)row[got.token] - (double)w.top) * a.s - log_d(w.sum));
            }
        }
    }
    if (!found) got = draw_from<T>(row, a.vocab, a.c, a.s, table, d.mode == kWithout ? d.x : -1, v);
    if ((threadIdx.x & 63) == 0) {
        const int64_t out = i * (a.drafts + 1) + d.t;
        a.tokens[out] = got.token;
        a.logp[out] = got.logp;
        a.count[i] = d.t + (got.token >= 0 ? 1 : 0);
    }
}

// Where a request's first token that is not accepted is, the sums of max(p - q, 0) there, and its last token.  Every workgroup of a request finds
// out the first for itself, and the last to be done the third (its sums are read in their own order, whichever that is): a launch each less.
template <typename T>
__global__ __launch_bounds__(kDrawBlock) void k_verify_rest(VerifyArgs a, int64_t first, int pieces, int64_t most, const BlockSum* target,
                                                            const BlockSum* draft, double* rest, unsigned* tickets) {
    __shared__ int last;
    const int64_t i = first + blockIdx.x / (unsigned)pieces;
    const int piece = blockIdx.x % (unsigned)pieces;
    const Decision d = decide<T>(a, i, most, target, draft, piece == 0);
    if (d.t < 0) return;
    if (d.mode != kRest) {
        if (piece == 0 && threadIdx.x < 64) finish<T>(a, i, d, most, target, nullptr);
        return;
    }
    double* sums = rest + i * most;
    const Line<T> line(row_of<T>(a.target, i, d.t), a.vocab);
    const T* drow = row_of<T>(a.draft, i, d.t);
    const int blocks = line.blocks(), each = (blocks + pieces - 1) / pieces, end = min((piece + 1) * each, blocks);
    for (int b = piece * each + (int)(threadIdx.x >> 6); b < end; b += kDrawWaves) {
        float v[Line<T>::kEntries];
        rest_of<T, true>(line, drow, b, a, d, v);
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < Line<T>::kEntries; ++e) sum += v[e];
        const double s = wave_sum((double)sum);
        if ((threadIdx.x & 63) == 0) publish(&sums[b], s);
    }
    if (!arrive_is_last(&tickets[i], &last, (unsigned)pieces)) return;
    if (threadIdx.x < 64) finish<T>(a, i, d, most, target, sums);
}

// The same without a drafter's rows.
template <typename T>
__global__ __launch_bounds__(kDrawBlock) void k_verify_draw(VerifyArgs a, int64_t first, int64_t most, const BlockSum* target) {
    const int64_t i = first + blockIdx.x;
    const Decision d = decide<T>(a, i, most, target, nullptr, true);
    if (d.t >= 0 && threadIdx.x < 64) finish<T>(a, i, d, most, target, nullptr);
}

constexpr int64_t kWorkgroupsMax = 1 << 22;      // of a launch (which takes fewer than 2^32 threads): longer batches take several

// Pieces of each of `rows` rows: enough workgroups to fill the card, as far as each of their waves has a block.
int pieces_of(int64_t rows, int64_t blocks, int64_t workgroups) {
    const int64_t want = (workgroups + rows - 1) / rows, most = (blocks + kDrawWaves - 1) / kDrawWaves;
    return (int)(want < most ? want : most);
}

// f(first, count): workgroups of `each` for rows first .. first + count - 1
template <typename F>
hipError_t in_launches(int64_t rows, int64_t each, F f) {
    const int64_t most = kWorkgroupsMax / each;
    for (int64_t r = 0; r < rows; r += most) {
        f(r, rows - r < most ? rows - r : most);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Waves that take a row together; 0: it is split over workgroups.
int row_waves(int64_t rows, int64_t blocks) {
    if (rows <= 64 && blocks > 64) return 0;
    const int64_t want = rows >= 2048 ? 4 : (rows >= 512 ? 8 : 16);
    return (int)(want < blocks ? want : blocks);
}

template <typename T>
hipError_t draw_rows(const DrawArgs& a, void* ws, hipStream_t st) {
    const int64_t most = blocks_of(a.vocab, sizeof(T));
    const int waves = row_waves(a.rows, most);
    if (waves)
        return in_launches(a.rows, 1, [&](int64_t first, int64_t n) {
            hipLaunchKernelGGL(k_draw_rows<T>, dim3((unsigned)n), dim3(waves * 64), most * sizeof(BlockSum), st, a, first);
        });
    const int pieces = pieces_of(a.rows, most, 2048);
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
    const bool rest = a.draft.z != nullptr, sums = rest && !a.draft_logp;
    const VerifySpace sp = verify_space(n, a.drafts, a.vocab, sizeof(T), rest, sums);
    char* at = (char*)ws;
    BlockSum *target = (BlockSum*)(at + sp.target), *draft = (BlockSum*)(at + sp.draft);
    double* parts = (double*)(at + sp.rest);
    unsigned* tickets = rest ? (unsigned*)(at + sp.tickets) : nullptr;
    const int64_t rows = n * a.target.each + (sums ? n * a.draft.each : 0);
    int pieces = pieces_of(rows, most, 4096);
    hipError_t e = in_launches(rows, pieces, [&](int64_t first, int64_t c) {
        hipLaunchKernelGGL(k_verify_sums<T>, dim3((unsigned)(c * pieces)), dim3(kDrawBlock), 0, st, a, first, pieces, most, target, draft, tickets);
    });
    if (e != hipSuccess) return e;
    if (!rest)
        return in_launches(n, 1, [&](int64_t first, int64_t c) {
            hipLaunchKernelGGL(k_verify_draw<T>, dim3((unsigned)c), dim3(kDrawBlock), 0, st, a, first, most, (const BlockSum*)target);
        });
    pieces = pieces_of(n, most, 1024);
    return in_launches(n, pieces, [&](int64_t first, int64_t c) {
        hipLaunchKernelGGL(k_verify_rest<T>, dim3((unsigned)(c * pieces)), dim3(kDrawBlock), 0, st, a, first, pieces, most, (const BlockSum*)target,
                           (const BlockSum*)draft, parts, tickets);
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

VerifySpace verify_space(int64_t requests, int64_t drafts, int64_t vocab, int size, bool draft_rows, bool draft_sums) {
    const size_t most = (size_t)blocks_of(vocab, size), n = (size_t)requests;
    VerifySpace s;
    s.target = 0;
    s.draft = rounded(n * (drafts + 1) * most * sizeof(BlockSum));
    s.rest = s.draft + (draft_sums ? rounded(n * drafts * most * sizeof(BlockSum)) : 0);
    s.tickets = s.rest + (draft_rows ? rounded(n * most * sizeof(double)) : 0);
    s.whole = s.tickets + (draft_rows ? rounded(n * sizeof(unsigned)) : 0);
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
