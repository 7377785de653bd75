// Tokens drawn from rows of logits by given numbers, and drafted tokens verified against the target's rows.
//
// A token is the first entry at which the running sum of p passes u.  With e_j = 2^((z_j - ref) c) a row is read once, in blocks of
// 2 kB whose sums are kept (8 bytes a block: 0.4 % of the row); in 64 bits the blocks' sums tell the block in which u S is
// passed, S being the whole row's, and that block alone is read again, lane by lane and entry by entry.  Sums of a block are in 32 bits and off by
// 2^-24 of the block's own, all else is in 64 bits.
//
// Verification: sums of all the target's rows (and of the drafter's, where its log-probabilities are not at hand) in one launch; the first
// token that is not accepted follows from them; at it, blocks of max(p - q, 0) are summed in a second launch, and a third finds the token.
#include "draws.h"

namespace lb {

namespace {

constexpr int kDrawBlock = 256, kDrawWaves = kDrawBlock / 64;

// 2^((z - ref) c) as it enters the sums of blocks.  (Both parts of the factor: the first alone would weigh entries far below the largest
// wrongly, by 3e-7 at 15 powers of two, all to one side.  The second takes no part where it is small against a distance without end.)
__device__ __forceinline__ float share(float z, float ref, Factor c) {
    const float d = z - ref;
    return exp2_hw(fmaf(d, c.c, fmaxf(d, -1000.0f) * c.low));
}
// The same with the rounding of the exponent put right: for differences p - q, and references that are not the largest.
__device__ __forceinline__ float share_exact(float z, float ref, Factor c) {
    const float d = z - ref, a = d * c.c, e = exp2_hw(a);
    const float rest = a > -1000.0f && a < 1000.0f ? fmaf(d, c.low, fmaf(d, c.c, -a)) : 0.0f;
    return fmaf(e, rest * 0.693147181f, e);
}

// A row as it is read in blocks: chunks of 16 bytes on boundaries of the logits, of which the first and the last may hold less of the row.
template <typename T>
struct Line {
    static constexpr int E = Chunk<T>::E, kPer = kBlockBytes / 16;
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
    // The lane's two chunks of block b.  A chunk that is not whole in the row is asked for as the nearest whole one, and mended below: no
    // branch stands around the loads.
    __device__ __forceinline__ void fetch(int b, int lane, vec (&v)[2]) const {
        if (high < low) return;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = min(max(b * kPer + k * 64 + lane, low), high);
            v[k] = *(const vec*)(row + first(i));
        }
    }
    __device__ __forceinline__ void mend(int b, int lane, vec (&v)[2]) const {
        if (b * kPer >= low && (b + 1) * kPer - 1 <= high) return;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = b * kPer + k * 64 + lane;
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
__device__ __forceinline__ void sum_blocks(const Line<T>& line, Factor c, int first, int end, int step, BlockSum* out) {
    constexpr int E = Line<T>::E;
    typedef typename Line<T>::vec vec;
    const int lane = threadIdx.x & 63;
    if (first >= end) return;
    float ref = -INFINITY;
    vec next[2];
    line.fetch(first, lane, next);
    for (int b = first; b < end; b += step) {
        vec v[2] = {next[0], next[1]};
        if (b + step < end) line.fetch(b + step, lane, next);
        line.mend(b, lane, v);
        float z[2 * E];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) z[k * E + e] = (float)v[k][e];
        float top = z[0];
#pragma unroll
        for (int e = 1; e < 2 * E; ++e) top = fmaxf(top, z[e]);
        if (__any(top > ref)) ref = fmaxf(ref, wave_max_f(top));
        const float at = anchor(ref);
#pragma unroll
        for (int e = 0; e < 2 * E; ++e) z[e] = share(z[e], at, c);
#pragma unroll
        for (int w = 1; w < 2 * E; w *= 2)
#pragma unroll
            for (int e = 0; e + w < 2 * E; e += 2 * w) z[e] += z[e + w];
        const float sum = wave_sum_f(z[0]);
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
    float top = -INFINITY;
    for (int b = lane; b < blocks; b += 64) top = fmaxf(top, table[b].ref);
    top = wave_max_f(top);
    double sum = 0.0;
    for (int b = lane; b < blocks; b += 64) sum += (double)table[b].sum * (double)weight_of(table[b].ref, top, c);
    return {top, wave_sum(sum)};
}

__device__ __forceinline__ double wave_running(double v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double w = __shfl_up(v, d);
        if (lane >= d) v += w;
    }
    return v;
}
__device__ __forceinline__ int last_lane(unsigned long long mask) { return 63 - __clzll(mask); }

// The block, of `blocks` with the sums at(b) >= 0, in which the running sum passes u of the whole, and how much of it is left there.  For all
// threads of a workgroup; total: the whole sum.  (Rounding can leave none that is passed: then it is the last block that has a share.  At least one
// has where total is above 0.)
struct Place {
    int block;
    double left, total;
};
struct WalkLds {
    double wave[kDrawWaves];
    Place place;
    int last[kDrawWaves];
};
template <typename At>
__device__ __forceinline__ Place find_block(int blocks, double u, WalkLds* lds, At at) {
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int each = (blocks + kDrawBlock - 1) / kDrawBlock, from = min(tid * each, blocks), to = min(from + each, blocks);
    double own = 0.0;
    for (int b = from; b < to; ++b) own += at(b);
    double running = wave_running(own);
    const unsigned long long some = __ballot(own > 0.0);
    if (lane == 63) lds->wave[wave] = running;
    if (lane == 0) lds->last[wave] = some ? wave * 64 + last_lane(some) : -1;
    __syncthreads();
    double before = 0.0, total = 0.0;
    int last = -1;
    for (int w = 0; w < kDrawWaves; ++w) {
        if (w < wave) before += lds->wave[w];
        total += lds->wave[w];
        last = max(last, lds->last[w]);
    }
    running += before;
    const double goal = u * total;
    // the first thread whose running sum passes the goal
    __syncthreads();
    const unsigned long long passed = __ballot(own > 0.0 && running > goal);
    if (lane == 0) lds->last[wave] = passed ? wave * 64 + __ffsll(passed) - 1 : -1;
    __syncthreads();
    int who = last;
    for (int w = kDrawWaves - 1; w >= 0; --w)
        if (lds->last[w] >= 0) who = lds->last[w];
    if (tid == who) {
        double sum = running - own, left = 0.0;
        int found = from;
        for (int b = from; b < to; ++b) {
            const double v = at(b);
            if (!(v > 0.0)) continue;
            found = b;
            left = goal - sum;
            sum += v;
            if (sum > goal) break;
        }
        lds->place = {found, fmax(left, 0.0), total};
    }
    __syncthreads();
    Place p = lds->place;
    if (who < 0) p = {-1, 0.0, total};
    return p;
}

// The entry, of a wave's 2 E a lane (z[k][e]: chunk k * 64 + lane), whose running sum passes `left`; its number in the block, -1 if none has a share.
template <int E>
__device__ __forceinline__ int find_entry(const float (&v)[2][E], double left) {
    double part[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        part[k] = 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) part[k] += (double)v[k][e];
    }
    double run[2] = {wave_running(part[0]), wave_running(part[1])};
    run[1] += __shfl(run[0], 63);
    int k = 0, who = -1;
    const unsigned long long p0 = __ballot(part[0] > 0.0 && run[0] > left), p1 = __ballot(part[1] > 0.0 && run[1] > left);
    const unsigned long long s0 = __ballot(part[0] > 0.0), s1 = __ballot(part[1] > 0.0);
    if (p0) who = __ffsll(p0) - 1;
    else if (p1) k = 1, who = __ffsll(p1) - 1;
    else if (s1) k = 1, who = last_lane(s1);
    else if (s0) who = last_lane(s0);
    if (who < 0) return -1;
    // (every lane looks among its own, the one in question tells)
    double sum = (k ? run[1] : run[0]) - (k ? part[1] : part[0]);
    int found = 0;
    bool done = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = k ? v[1][e] : v[0][e];
        if (x > 0.0f && !done) {
            found = e;
            sum += (double)x;
            done = sum > left;
        }
    }
    return (k * 64 + who) * E + __shfl(found, who);
}

// u in [0, 1)
__device__ __forceinline__ double number(float u) { return (double)fminf(fmaxf(u, 0.0f), 0x1.fffffep-1f); }

// ---- drawing from p ----------------------------------------------------------------------------------------------------------

struct Drawn {
    int token;
    float logp;
};

// Entry of p, without entry `skip` (-1: none is left out) where anything else has a share, by a whole workgroup; the first wave's lanes get it.
template <typename T>
__device__ __forceinline__ Drawn draw_from(const T* row, int vocab, Factor c, double s, const BlockSum* table, int skip, float u, WalkLds* lds,
                                           Whole* whole_lds) {
    const Line<T> line(row, vocab);
    constexpr int E = Line<T>::E;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, blocks = line.blocks();
    auto entries = [&](int b, float ref, int without, float (&v)[2][E]) {
        typename Line<T>::vec raw[2];
        line.fetch(b, lane, raw);
        line.mend(b, lane, raw);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool gone = line.first(b * Line<T>::kPer + k * 64 + lane) + e == without;
                v[k][e] = gone ? 0.0f : share((float)raw[k][e], anchor(ref), c);
            }
    };
    __shared__ float skipped;            // the sum of the block that is short of an entry
    if (wave == 0) {
        const Whole w = wave_whole(table, blocks, c);
        if (lane == 0) *whole_lds = w;
        if (skip >= 0) {
            float v[2][E];
            const int b = line.block_of(skip);
            entries(b, table[b].ref, skip, v);
            float sum = 0.0f;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) sum += v[k][e];
            sum = wave_sum_f(sum);
            if (lane == 0) skipped = sum;
        }
    }
    __syncthreads();
    const Whole w = *whole_lds;
    if (!(w.sum > 0.0 && w.sum < INFINITY) || u != u) return {-1, NAN};
    auto at = [&](int b) {
        const float sum = skip >= 0 && b == line.block_of(skip) ? skipped : table[b].sum;
        return (double)sum * (double)weight_of(table[b].ref, w.top, c);
    };
    Place p = find_block(blocks, number(u), lds, at);
    if (p.block < 0) {                   // (nothing else has a share: with the entry that was to be left out)
        skip = -1;
        __syncthreads();
        p = find_block(blocks, number(u), lds, at);
    }
    if (wave != 0) return {};
    const float ref = table[p.block].ref;
    float v[2][E];
    entries(p.block, ref, skip, v);
    const int found = find_entry<E>(v, p.left / (double)weight_of(ref, w.top, c));
    if (found < 0) return {-1, NAN};
    const int token = line.first(p.block * Line<T>::kPer) + found;
    return {token, (float)(((double)(float)row[token] - (double)w.top) * s - log_d(w.sum))};
}

template <typename T>
__global__ __launch_bounds__(kDrawBlock) void k_block_sums(const T* z, int64_t ld, int vocab, Factor c, int64_t first, int pieces, int64_t most,
                                                           BlockSum* table) {
    const int64_t r = first + blockIdx.x / (unsigned)pieces;
    const Line<T> line(z + r * ld, vocab);
    const int piece = blockIdx.x % (unsigned)pieces, blocks = line.blocks(), each = (blocks + pieces - 1) / pieces;
    sum_blocks<T>(line, c, piece * each + (int)(threadIdx.x >> 6), min((piece + 1) * each, blocks), kDrawWaves, table + r * most);
}

template <typename T>
__global__ __launch_bounds__(kDrawBlock) void k_draw(DrawArgs a, int64_t first, int64_t most, const BlockSum* table) {
    __shared__ WalkLds lds;
    __shared__ Whole whole;
    const int64_t r = first + blockIdx.x;
    const Drawn d = draw_from<T>((const T*)a.z + r * a.ld, a.vocab, a.c, a.s, table + r * most, -1, a.uniform[r], &lds, &whole);
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

// Sums of the rows that may be asked for: the target's (DRAFT: the drafter's) at positions up to (before) a request's length.
template <typename T, bool DRAFT>
__global__ __launch_bounds__(kDrawBlock) void k_verify_sums(VerifyArgs a, int64_t first, int pieces, int64_t most, BlockSum* table) {
    const RowSet& set = DRAFT ? a.draft : a.target;
    const int64_t r = first + blockIdx.x / (unsigned)pieces, i = r / set.each;
    const int t = (int)(r - i * set.each), n = length_of(a, i);
    if (n < 0 || t > n - (DRAFT ? 1 : 0)) return;
    const Line<T> line(row_of<T>(set, i, t), a.vocab);
    const int piece = blockIdx.x % (unsigned)pieces, blocks = line.blocks(), each = (blocks + pieces - 1) / pieces;
    sum_blocks<T>(line, DRAFT ? a.draft_c : a.c, piece * each + (int)(threadIdx.x >> 6), min((piece + 1) * each, blocks), kDrawWaves, table + r * most);
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
    const int64_t x = a.drafted[at];
    const T* row = row_of<T>(a.target, i, t);
    Verdict v = {0, 0.0f, {t, kFromTarget, 0, 0.0f, 0.0f, 0.0f, 0.0f}};
    if (x < 0 || x >= a.vocab) return v;
    const Whole p = wave_whole(target + (i * a.target.each + t) * most, Line<T>(row, a.vocab).blocks(), a.c);
    if (!(p.sum > 0.0 && p.sum < INFINITY)) return v;
    const double lp = ((double)(float)row[x] - (double)p.top) * a.s - log_d(p.sum);
    double q = 1.0;
    if (a.draft.z) {
        const T* drow = row_of<T>(a.draft, i, t);
        const float zx = (float)drow[x];
        if (a.draft_logp) {
            q = exp((double)a.draft_logp[at]);
            if (!(q > 0.0 && q < INFINITY && fabsf(zx) < INFINITY)) return v;
            v.next.q_ref = zx;
            v.next.q_factor = (float)q;
        } else {
            const Whole w = wave_whole(draft + (i * a.draft.each + t) * most, Line<T>(drow, a.vocab).blocks(), a.draft_c);
            if (!(w.sum > 0.0 && w.sum < INFINITY)) return v;
            q = exp(((double)zx - (double)w.top) * a.draft_s) / w.sum;
            v.next.q_ref = w.top;
            v.next.q_factor = (float)(1.0 / w.sum);
        }
        v.next.mode = kRest;
        v.next.m = p.top;
        v.next.inv = (float)(1.0 / p.sum);
    } else {
        v.next.mode = kWithout;
        v.next.x = (int)x;
    }
    v.accepted = q > 0.0 && (double)a.uniform[at] * q < exp(lp);
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
template <typename T>
__device__ __forceinline__ void rest_of(const Line<T>& line, const T* drow, int b, const VerifyArgs& a, const Decision& d, float (&v)[2][Line<T>::E]) {
    const int lane = threadIdx.x & 63;
    typename Line<T>::vec p[2], q[2];
    line.fetch(b, lane, p);
#pragma unroll
    for (int k = 0; k < 2; ++k) q[k] = line.beside(drow, b * Line<T>::kPer + k * 64 + lane);
    line.mend(b, lane, p);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < Line<T>::E; ++e) {
            const float r = share_exact((float)p[k][e], d.m, a.c) * d.inv - share_exact((float)q[k][e], d.q_ref, a.draft_c) * d.q_factor;
            v[k][e] = r <= 0.0f ? 0.0f : r;
        }
}

// Where a request's first token that is not accepted is, and the sums of max(p - q, 0) there.  Every workgroup of a request finds out
// the first for itself: a launch less.
template <typename T>
__global__ __launch_bounds__(kDrawBlock) void k_verify_rest(VerifyArgs a, int64_t first, int pieces, int64_t most, const BlockSum* target,
                                                            const BlockSum* draft, double* rest, Decision* decision) {
    const int64_t i = first + blockIdx.x / (unsigned)pieces;
    const int piece = blockIdx.x % (unsigned)pieces;
    const Decision d = decide<T>(a, i, most, target, draft, piece == 0);
    if (piece == 0 && threadIdx.x == 0) decision[i] = d;
    if (d.t < 0 || d.mode != kRest) return;
    const Line<T> line(row_of<T>(a.target, i, d.t), a.vocab);
    const T* drow = row_of<T>(a.draft, i, d.t);
    const int blocks = line.blocks(), each = (blocks + pieces - 1) / pieces, end = min((piece + 1) * each, blocks);
    for (int b = piece * each + (int)(threadIdx.x >> 6); b < end; b += kDrawWaves) {
        float v[2][Line<T>::E];
        rest_of<T>(line, drow, b, a, d, v);
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int e = 0; e < Line<T>::E; ++e) sum += v[k][e];
        const double s = wave_sum((double)sum);
        if ((threadIdx.x & 63) == 0) rest[i * most + b] = s;
    }
}

// The last token of a request.
template <typename T>
__global__ __launch_bounds__(kDrawBlock) void k_verify_draw(VerifyArgs a, int64_t first, int64_t most, const BlockSum* target, const BlockSum* draft,
                                                            const double* rest, const Decision* decision) {
    __shared__ WalkLds lds;
    __shared__ Whole whole;
    const int64_t i = first + blockIdx.x;
    const Decision d = decision ? decision[i] : decide<T>(a, i, most, target, draft, true);
    if (d.t < 0) return;
    const T* row = row_of<T>(a.target, i, d.t);
    const BlockSum* table = target + (i * a.target.each + d.t) * most;
    const float v = a.last_uniform[i];
    Drawn got = {-1, NAN};
    bool found = false;
    if (d.mode == kRest && v == v) {
        const Line<T> line(row, a.vocab);
        const double* sums = rest + i * most;
        // (a sum that is no number makes the total one: p is drawn from)
        const Place p = find_block(line.blocks(), number(v), &lds, [&](int b) { return sums[b]; });
        if (p.block >= 0 && p.total > 0.0 && p.total < INFINITY) {
            found = true;
            if (threadIdx.x < 64) {
                float part[2][Line<T>::E];
                rest_of<T>(line, row_of<T>(a.draft, i, d.t), p.block, a, d, part);
                const int e = find_entry<Line<T>::E>(part, p.left);
                const Whole w = wave_whole(table, line.blocks(), a.c);
                if (e >= 0) {
                    got.token = line.first(p.block * Line<T>::kPer) + e;
                    got.logp = (float)(((double)(float)row[got.token] - (double)w.top) * a.s - log_d(w.sum));
                }
            }
        }
        __syncthreads();
    }
    if (!found) got = draw_from<T>(row, a.vocab, a.c, a.s, table, d.mode == kWithout ? d.x : -1, v, &lds, &whole);
    if (threadIdx.x == 0) {
        const int64_t out = i * (a.drafts + 1) + d.t;
        a.tokens[out] = got.token;
        a.logp[out] = got.logp;
        a.count[i] = d.t + (got.token >= 0 ? 1 : 0);
    }
}

constexpr int64_t kWorkgroupsMax = 1 << 23;      // of a launch (which takes fewer than 2^32 threads): longer batches take several

// Pieces of each of `rows` rows, so that there are about as many workgroups as keep the card busy; one at least has a block for each wave.
int pieces_of(int64_t rows, int64_t blocks) {
    const int64_t want = (2048 + rows - 1) / rows, most = (blocks + kDrawWaves - 1) / kDrawWaves;
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

template <typename T>
hipError_t draw_rows(const DrawArgs& a, void* ws, hipStream_t st) {
    const int64_t most = blocks_of(a.vocab, sizeof(T));
    const int pieces = pieces_of(a.rows, most);
    BlockSum* table = (BlockSum*)ws;
    hipError_t e = in_launches(a.rows, pieces, [&](int64_t first, int64_t n) {
        hipLaunchKernelGGL(k_block_sums<T>, dim3((unsigned)(n * pieces)), dim3(kDrawBlock), 0, st, (const T*)a.z, a.ld, a.vocab, a.c, first, pieces, most, table);
    });
    if (e != hipSuccess) return e;
    return in_launches(a.rows, 1, [&](int64_t first, int64_t n) {
        hipLaunchKernelGGL(k_draw<T>, dim3((unsigned)n), dim3(kDrawBlock), 0, st, a, first, most, (const BlockSum*)table);
    });
}

template <typename T>
hipError_t verify_rows(const VerifyArgs& a, void* ws, hipStream_t st) {
    const int64_t most = blocks_of(a.vocab, sizeof(T)), n = a.requests;
    const bool sums = a.draft.z && !a.draft_logp && a.drafts > 0, rest = a.draft.z && a.drafts > 0;
    const VerifySpace sp = verify_space(n, a.drafts, a.vocab, sizeof(T), rest, sums);
    char* at = (char*)ws;
    BlockSum *target = (BlockSum*)(at + sp.target), *draft = (BlockSum*)(at + sp.draft);
    double* parts = (double*)(at + sp.rest);
    Decision* decision = (Decision*)(at + sp.decision);
    hipError_t e = hipSuccess;
    {
        const int64_t rows = n * a.target.each;
        const int pieces = pieces_of(rows, most);
        e = in_launches(rows, pieces, [&](int64_t first, int64_t c) {
            hipLaunchKernelGGL((k_verify_sums<T, false>), dim3((unsigned)(c * pieces)), dim3(kDrawBlock), 0, st, a, first, pieces, most, target);
        });
        if (e != hipSuccess) return e;
    }
    if (sums) {
        const int64_t rows = n * a.draft.each;
        const int pieces = pieces_of(rows, most);
        e = in_launches(rows, pieces, [&](int64_t first, int64_t c) {
            hipLaunchKernelGGL((k_verify_sums<T, true>), dim3((unsigned)(c * pieces)), dim3(kDrawBlock), 0, st, a, first, pieces, most, draft);
        });
        if (e != hipSuccess) return e;
    }
    if (rest) {
        const int pieces = pieces_of(n, most);
        e = in_launches(n, pieces, [&](int64_t first, int64_t c) {
            hipLaunchKernelGGL(k_verify_rest<T>, dim3((unsigned)(c * pieces)), dim3(kDrawBlock), 0, st, a, first, pieces, most, (const BlockSum*)target,
                               (const BlockSum*)draft, parts, decision);
        });
        if (e != hipSuccess) return e;
    }
    return in_launches(n, 1, [&](int64_t first, int64_t c) {
        hipLaunchKernelGGL(k_verify_draw<T>, dim3((unsigned)c), dim3(kDrawBlock), 0, st, a, first, most, (const BlockSum*)target, (const BlockSum*)draft,
                           (const double*)parts, (const Decision*)(rest ? decision : nullptr));
    });
}

template <typename F>
hipError_t by_type(int dtype, F f) {
    return dtype == LBFGSB_F32 ? f(float{}) : (dtype == LBFGSB_BF16 ? f(__bf16{}) : f(_Float16{}));
}

size_t rounded(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

size_t draw_space(int64_t rows, int64_t vocab, int size) { return rounded((size_t)(rows * blocks_of(vocab, size)) * sizeof(BlockSum)); }

VerifySpace verify_space(int64_t requests, int64_t drafts, int64_t vocab, int size, bool draft_rows, bool draft_sums) {
    const size_t most = (size_t)blocks_of(vocab, size), n = (size_t)requests;
    VerifySpace s;
    s.target = 0;
    s.draft = rounded(n * (drafts + 1) * most * sizeof(BlockSum));
    s.rest = s.draft + (draft_sums ? rounded(n * drafts * most * sizeof(BlockSum)) : 0);
    s.decision = s.rest + (draft_rows ? rounded(n * most * sizeof(double)) : 0);
    s.whole = s.decision + (draft_rows ? rounded(n * sizeof(Decision)) : 0);
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
