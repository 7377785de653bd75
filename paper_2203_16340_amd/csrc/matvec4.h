// Products y = x W^T of a few rows x with weights of 4 bits.  Included once for each type of x.
//
// With w = scale (code - zero) a group's part of a product is scale (sum_j code_j x_j - zero sum_j x_j).  Codes are whole numbers of 4 bits, exact in
// bf16 and f16, so the first sum is matrix instructions on the codes themselves, with exact products and sums in 32 bits; the second is formed once
// for all rows of W, and scale and zero enter once a group.  x in 32 bits goes in as three bf16 parts, which hold its 24 bits.
//
// Bound by memory: half a byte and one or two instructions a weight.  A code becomes a matrix operand in 7/8 of an instruction: a byte
// 0 .. 15 is, read as an 8-bit float with 3 bits of mantissa, that number times 2^-9 (denormal below 8, the first binade from there), so masking
// the two halves of a word and four conversions of pairs with a scale of 2^9 make eight of them.
#pragma once

#include "weights4.h"

namespace lb {

namespace {

typedef unsigned int u4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Operand;
template <>
struct Operand<__bf16> {
    typedef __bf16 vec __attribute__((ext_vector_type(8)));
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ pair codes(unsigned v, bool high) {
        return high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 512.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, 512.0f, false);
    }
    static __device__ __forceinline__ f4 product(vec a, vec b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Operand<_Float16> {
    typedef _Float16 vec __attribute__((ext_vector_type(8)));
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ pair codes(unsigned v, bool high) {
        return high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 512.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 512.0f, false);
    }
    static __device__ __forceinline__ f4 product(vec a, vec b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <typename T>
struct OperandOf { typedef T type; };
template <>
struct OperandOf<float> { typedef __bf16 type; };

// eight codes as an operand, in the order of their columns
template <typename M>
__device__ __forceinline__ typename Operand<M>::vec unpacked(unsigned word) {
    const unsigned low = word & 0x0f0f0f0fu, high = (word >> 4) & 0x0f0f0f0fu;
    const auto a = Operand<M>::codes(low, false), b = Operand<M>::codes(low, true), c = Operand<M>::codes(high, false), d = Operand<M>::codes(high, true);
    return {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight entries of x as operands: itself, or its bf16 parts.
template <typename X>
struct Parts {
    static constexpr int N = 1;
    typedef typename Operand<X>::vec vec;
    vec p[1];
    __device__ __forceinline__ void set(const X (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) p[0][e] = x[e];
    }
};
template <>
struct Parts<float> {
    static constexpr int N = 3;
    typedef Operand<__bf16>::vec vec;
    vec p[3];
    __device__ __forceinline__ void set(const float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // (each difference is exact; an infinite x leaves NaN behind it, and so does one that rounds to infinity)
            const __bf16 a = (__bf16)x[e];
            const float r = x[e] - (float)a;
            const __bf16 b = (__bf16)r;
            p[0][e] = a;
            p[1][e] = b;
            p[2][e] = (__bf16)(r - (float)b);
        }
    }
};

// NT scales that stand side by side.  As uint16_t they are the bits of bf16 or f16, and which is asked at each, two instructions more: one kernel for both where
// x is laid out, and where W has fewer than 256 blocks, which the compiler takes a third less time for (65536 x 4096 with 48 rows 50.3 us, with kernels of
// their own 50.2).  With more blocks and x in LDS from the start each type has its own (one row with 131072 x 4096 43.9 us for 44.6, 5 with 50021 x 2600 17.5 for 18.0).
template <typename S, int NT>
struct Scales {
    typedef S vec __attribute__((ext_vector_type(NT)));
};
template <typename S>
__device__ __forceinline__ float scale_of(S s, bool) { return (float)s; }
template <>
__device__ __forceinline__ float scale_of<uint16_t>(uint16_t s, bool bf16) {
    return bf16 ? __builtin_bit_cast(float, (uint32_t)s << 16) : (float)__builtin_bit_cast(_Float16, s);
}

// What a launch is made of: waves of a workgroup that take rows beside each other, and waves that share their steps.
struct Shape {
    int row_waves, step_waves;
    int chunk_log2;          // steps of x that are in LDS at a time: at least one for each of the waves that share them
};
constexpr int row_waves_of(int T) { return T == 1 ? 1 : 4; }     // the least

// x as operands, step by step, in units of 16 bytes (eight columns of a row): for each of a step's four instructions its four such, and for each of those the
// rows one behind the other, so that 16 lanes read 256 bytes.  A 32-bit x is three planes of that.  Where x is laid out beforehand the rows are filled up to
// 16 T, and behind a step's operands stand the sums of x over its groups, or over its part of one: 4 / G times 16 T floats, in the order of the
// result registers.
template <typename X>
__host__ __device__ constexpr int operand_units(int rows) { return Parts<X>::N * 16 * rows; }
template <typename X>
__host__ __device__ constexpr int step_units(int G, int T) { return operand_units<X>(16 * T) + 16 / G * T; }
__device__ __forceinline__ int unit_at(int part, int j, int kq, int rows, int row) { return ((part * 4 + j) * 4 + kq) * rows + row; }

// (no wait for loads from memory, which stay on their way over it)
__device__ __forceinline__ void barrier_for_lds() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
// The thread's index, to the compiler a new value each time: else it keeps the addresses of all that a thread brings to LDS, single entries too,
// over the loop, some 100 registers.
__device__ __forceinline__ int fresh_thread() {
    int t = (int)threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// eight entries of a row from column col on, 0 past its end
template <typename X>
__device__ __forceinline__ void eight(const X* row, int col, int cols, bool some, X (&v)[8]) {
    typedef X wide __attribute__((ext_vector_type(8), aligned(sizeof(X))));
    if (some && col + 8 <= cols) {
        const wide w = *(const wide*)(row + col);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = w[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = some && col + e < cols ? row[col + e] : (X)0.0f;
    }
}

// All of x's (up to 16) rows to LDS, by a whole workgroup, N units of a thread on their way at once.
template <typename X, int N>
__device__ __forceinline__ void bring_by(const Matvec4Args& a, int64_t x0, int rows, typename Operand<typename OperandOf<X>::type>::vec* lds) {
    const int tid = threadIdx.x, kq = tid & 3, j = (tid >> 2) & 3, steps = a.w.steps(), stride = (int)blockDim.x >> 4, units = operand_units<X>(rows);
    int row = 0, step = tid >> 4;
    auto settle = [&] {
        while (step >= steps) {
            step -= steps;
            ++row;
        }
    };
    settle();
    while (row < rows) {
        X v[N][8];
        int to[N];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const bool some = row < rows;
            to[k] = some ? step * units + unit_at(0, j, kq, rows, row) : -1;
            eight((const X*)a.x + (x0 + (some ? row : 0)) * a.ld_x, step * kStepCols + 32 * j + 8 * kq, a.w.cols, some, v[k]);
            step += stride;
            settle();
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (to[k] < 0) continue;
            Parts<X> p;
            p.set(v[k]);
#pragma unroll
            for (int n = 0; n < Parts<X>::N; ++n) lds[to[k] + n * 16 * rows] = p.p[n];
        }
    }
}
// (With a block of W to a workgroup, 50021 x 2600 with 5 rows of f16 waited four times two at a time, and twice four at a time: 20.8 us, with eight 19.8.  But eight where there are
// two cost 131072 x 4096 with one row 47.9 us for 44.9.)
template <typename X>
__device__ __forceinline__ void bring_whole(const Matvec4Args& a, int64_t x0, int rows, typename Operand<typename OperandOf<X>::type>::vec* lds) {
    const int all = rows * a.w.steps(), stride = (int)blockDim.x >> 4;      // a thread's units: all / stride
    if (all <= 2 * stride) bring_by<X, 2>(a, x0, rows, lds);
    else if (sizeof(X) == 4 || all <= 4 * stride) bring_by<X, 4>(a, x0, rows, lds);
    else if constexpr (sizeof(X) == 2) bring_by<X, 8>(a, x0, rows, lds);
}

// What brings x, laid out by k_operands4, to LDS a few steps at a time; a thread's units of the next are on their way while these are used.
// (Laid out by every workgroup for itself, 65536 x 4096 with 48 rows took 83 us: more instructions than the products.)
template <typename X, int G, int T>
struct LaidOut {
    typedef typename Operand<typename OperandOf<X>::type>::vec vec;
    static constexpr int kUnits = step_units<X>(G, T), kPieces = (kUnits + 64 * row_waves_of(T) - 1) / (64 * row_waves_of(T));   // (a step a wave)
    vec piece[kPieces];
    __device__ __forceinline__ void load(const Matvec4Args& a, int64_t x0, int first, int chunk_log2) {
        const int steps = a.w.steps();
        const vec* from = (const vec*)a.operands + (x0 / (16 * T) * steps + first) * kUnits;
        const int most = min(1 << chunk_log2, steps - first) * kUnits - 1, tid = fresh_thread();
#pragma unroll
        for (int k = 0; k < kPieces; ++k) piece[k] = from[min(tid + k * (int)blockDim.x, most)];
    }
    __device__ __forceinline__ void store(vec* lds, int chunk_log2) const {
        const int all = kUnits << chunk_log2, tid = fresh_thread();
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
            if (tid + k * (int)blockDim.x < all) lds[tid + k * (int)blockDim.x] = piece[k];
    }
};

// A thread for eight entries of x.
template <typename X, int G, int T>
__global__ __launch_bounds__(256) void k_operands4(Matvec4Args a) {
    typedef typename Operand<typename OperandOf<X>::type>::vec vec;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, at = i >> 4;
    const int steps = a.w.steps(), kq = (int)i & 3, j = (int)(i >> 2) & 3;
    const int64_t token = at / steps, pass = token / (16 * T);
    if (token >= a.tokens) return;              // (16 lanes at a time: they share a row's step)
    const int step = (int)(at - token * steps), row = (int)(token - pass * (16 * T));
    X v[8];
    eight((const X*)a.x + token * a.ld_x, step * kStepCols + 32 * j + 8 * kq, a.w.cols, true, v);
    vec* to = (vec*)a.operands + (pass * steps + step) * step_units<X>(G, T);
    Parts<X> p;
    p.set(v);
#pragma unroll
    for (int n = 0; n < Parts<X>::N; ++n) to[unit_at(n, j, kq, 16 * T, row)] = p.p[n];
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += (float)v[e];
    sum += dpp_move_f<kDppXor1>(sum);
    sum += dpp_move_f<kDppXor2>(sum);
    if (G >= 2) sum += dpp_move_f<kDppHalfMirror>(sum);
    if (G == 4) sum += dpp_move_f<kDppMirror>(sum);
    if (kq == 0 && j % G == 0) ((float*)(to + operand_units<X>(16 * T)))[j / G * (16 * T) + (row & ~15) + 4 * (row & 3) + ((row >> 2) & 3)] = sum;
}

// A wave's share of up to 16 T rows of x against NT tiles of a block.  The waves' sums are joined in LDS in a fixed order.
// x's row i of 16 stands at row 4 (i % 4) + i / 4 of the operand, so that up to four rows take one of the four result registers; where there are
// fewer rows the rest of the operand is anything, and what comes of it is not looked at.
// S: the scales' type.  WHOLE: all of x is in LDS from the start, and x has up to 16 rows.
// One row with 131072 x 4096 takes 43.8 us, 6.3 TB/s (loads without products 42.8).  Below some 100 MB it is what comes before the first product and behind the
// last that counts, 7 to 9 us: 50021 x 2600 with 5 rows 17.5.  65536 x 4096 with 48 rows 47 behind k_operands4's 3.3: LDS, 24 000 of
// 100 000 cycles, and waits at its barriers.
// Waves a unit: as many, up to four, as the registers allow without spills.  With two matrix instructions a group and 32-bit scales or 32-bit x it takes 132 to 152 of them, which four
// waves do not have (16 to 152 bytes a lane would be spilled), x laid out first 136 to 156; x in 32 bits laid out, and more than one tile, up to 256.
template <typename X, typename S, int G, int NT, int T, bool WHOLE>    // G: matrix instructions between two groups, 1, 2 or 4
__global__ __launch_bounds__(512, T > 1 || (!WHOLE && sizeof(X) == 4) ? 2 : (WHOLE && (G != 2 || sizeof(S) + sizeof(X) < 6) ? 4 : 3)) void k_matvec4(Matvec4Args a, Shape shape) {
    extern __shared__ char shared[];
    typedef typename OperandOf<X>::type M;
    typedef typename Operand<M>::vec vec;
    typedef typename Scales<S, NT>::vec SN;
    constexpr int kRows = 16 * NT, kParts = Parts<X>::N;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, kq = lane >> 4;
    const int row_wave = wave % shape.row_waves, waves = shape.step_waves, part = wave / shape.row_waves;
    const int64_t units = a.w.blocks() * (4 / NT), first_unit = (int64_t)blockIdx.x * shape.row_waves;      // of NT tiles
    const int64_t unit = first_unit + row_wave < units ? first_unit + row_wave : units - 1, block = unit / (4 / NT);
    const int tile = (int)(unit % (4 / NT)) * NT;
    const int64_t x0 = (int64_t)blockIdx.y * (16 * T);
    const int have = (int)(a.tokens - x0 < 16 * T ? a.tokens - x0 : 16 * T);
    const int steps = a.w.steps(), groups = a.w.groups(), chunk = 1 << shape.chunk_log2;
    const char* codes = (const char*)a.packed + (size_t)block * steps * kStepBytes + tile * kTileBytes + lane * 16;
    const S* scales = (const S*)((const char*)a.packed + a.w.code_bytes()) + (size_t)block * groups * kBlockRows * (1 + a.w.zeros) + 4 * c + tile;
    const int each = kBlockRows * (1 + a.w.zeros);
    const bool bf16 = a.w.scale_type == LBFGSB_BF16;

    f4 y[NT][T];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int u = 0; u < T; ++u) y[t][u] = f4{0.0f, 0.0f, 0.0f, 0.0f};

    struct Step {
        u4 w[NT];
        SN scale[4 / G], zero[4 / G];
    };
    auto load = [&](Step& st, int s) {
#pragma unroll
        for (int t = 0; t < NT; ++t) st.w[t] = __builtin_nontemporal_load((const u4*)(codes + (size_t)s * kStepBytes + t * kTileBytes));
#pragma unroll
        for (int g = 0; g < 4 / G; ++g) {
            // (a last group may end before its step does; what comes after it is 0 times the scale of a group that is there)
            const int at = min((s * kStepCols + g * G * 32) >> a.w.group_log2, groups - 1);
            const S* from = scales + (size_t)at * each;
            st.scale[g] = *(const SN*)from;
            if (a.w.zeros) st.zero[g] = *(const SN*)(from + kBlockRows);
        }
    };
    int row_at[T];
#pragma unroll
    for (int u = 0; u < T; ++u) row_at[u] = WHOLE ? kq * have + min(4 * (c & 3) + (c >> 2), have - 1) : kq * 16 * T + 16 * u + 4 * (c & 3) + (c >> 2);
    vec ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (M)1.0f;
    auto multiply = [&](const Step& st, const vec* in) {            // in: the step's operands
        const int rows = WHOLE ? have : 16 * T;
        const f4* totals = (const f4*)(in + operand_units<X>(16 * T));
        f4 sum[NT][T], all1;
        (void)totals;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (j % G == 0) {
#pragma unroll
                for (int u = 0; u < T; ++u)
#pragma unroll
                    for (int t = 0; t < NT; ++t) sum[t][u] = f4{0.0f, 0.0f, 0.0f, 0.0f};
                all1 = f4{0.0f, 0.0f, 0.0f, 0.0f};
            }
            // (or the compiler has the operands of all four at once, and spills)
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            vec w[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) w[t] = unpacked<M>(st.w[t][j]);
#pragma unroll
            for (int u = 0; u < T; ++u)
#pragma unroll
                for (int n = 0; n < kParts; ++n) {
                    const vec v = in[(n * 4 + j) * 4 * rows + row_at[u]];
                    // (the matrix unit has time for their sums as well)
                    if (WHOLE) all1 = Operand<M>::product(v, ones, all1);
#pragma unroll
                    for (int t = 0; t < NT; ++t) sum[t][u] = Operand<M>::product(v, w[t], sum[t][u]);
                }
            if (j % G == G - 1) {
                const int g = j / G;
#pragma unroll
                for (int u = 0; u < T; ++u) {
                    const f4 all = WHOLE ? all1 : totals[(g * T + u) * 4 + kq];
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const float scale = scale_of(st.scale[g][t], bf16), zero = a.w.zeros ? scale_of(st.zero[g][t], bf16) : 8.0f;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (T > 1 || r == 0 || have > 4) y[t][u][r] = fmaf(scale, fmaf(-zero, all[r], sum[t][u][r]), y[t][u][r]);
                    }
                }
            }
        }
    };

    // In turn i a wave takes step part + i * waves.  kDepth steps of codes are on their way at once; loads come back in order, so what is asked
    // for last must be needed last, and no branch stands around those of the main loop, or all of them would be waited for behind it.
    constexpr int kDepth = NT == 1 ? 4 : 2;
    const int turns = (steps + waves - 1) / waves;
    auto step_of = [&](int i) { return min(part + i * waves, steps - 1); };
    LaidOut<X, G, T> stage;
    vec* lds = (vec*)shared;
    const int per_step = WHOLE ? operand_units<X>(have) : step_units<X>(G, T), room = per_step << shape.chunk_log2;
    if (!WHOLE) stage.load(a, x0, 0, shape.chunk_log2);
    Step at[kDepth];
#pragma unroll
    for (int d = 0; d < kDepth; ++d) load(at[d], step_of(d));
    if (WHOLE) bring_whole<X>(a, x0, have, lds);
    else stage.store(lds, shape.chunk_log2);
    barrier_for_lds();
    int chunk_at = 0, half = 0;                                     // first step of the chunk in LDS, and where it is
    if (!WHOLE && chunk < steps) stage.load(a, x0, chunk, shape.chunk_log2);
    auto turn = [&](int i, const Step& st) {
        if (!WHOLE && i * waves >= chunk_at + chunk) {              // (all waves come to a chunk's end in the same turn: a chunk is a number of turns)
            half ^= 1;
            stage.store(lds + half * room, shape.chunk_log2);
            barrier_for_lds();
            chunk_at += chunk;
            if (chunk_at + chunk < steps) stage.load(a, x0, chunk_at + chunk, shape.chunk_log2);
        }
        const int s = part + i * waves;
        if (s < steps) multiply(st, lds + half * room + (s - chunk_at) * per_step);
    };
    int i = 0;
    for (; i + 2 * kDepth <= turns; i += kDepth) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            turn(i + d, at[d]);
            load(at[d], step_of(i + d + kDepth));
        }
    }
    for (; i < turns; i += kDepth) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            if (i + d < turns) turn(i + d, at[d]);
            if (i + d + kDepth < turns) load(at[d], step_of(i + d + kDepth));
        }
    }

    // register r holds row 4 r + kq of 16
    __syncthreads();
    float* sums = (float*)shared;
    const int all_rows = shape.row_waves * kRows;
#pragma unroll
    for (int u = 0; u < T; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 16 * u + 4 * r + kq;
            if (i < have) {
#pragma unroll
                for (int t = 0; t < NT; ++t) sums[(part * have + i) * all_rows + row_wave * kRows + NT * c + t] = y[t][u][r];
            }
        }
    __syncthreads();
    for (int k = threadIdx.x; k < have * all_rows; k += blockDim.x) {
        const int i = k / all_rows, o = k % all_rows;
        const int64_t of = first_unit + o / kRows, row = of / (4 / NT) * kBlockRows + o % kRows / NT * 4 + of % (4 / NT) * NT + o % NT;
        float sum = 0.0f;
        for (int w = 0; w < waves; ++w) sum += sums[w * have * all_rows + k];
        if (row < a.w.rows) {
            const int64_t to = (x0 + i) * a.ld_y + row;
            if (a.y_type == LBFGSB_F32) ((float*)a.y)[to] = sum;
            else ((X*)a.y)[to] = (X)sum;
        }
    }
}

template <typename X, typename S, int G, int NT, int T, bool WHOLE>
hipError_t matvec4_in(const Matvec4Args& a, int row_waves, int step_waves, hipStream_t st) {
    const int64_t units = a.w.blocks() * (4 / NT), steps = a.w.steps();
    const int have = a.tokens < 16 * T ? (int)a.tokens : 16 * T;
    while (step_waves > steps) step_waves /= 2;
    if (!WHOLE)                          // (a step a wave, twice: no more than a compute unit's LDS)
        while ((size_t)step_units<X>(G, T) * 16 * 2 * step_waves > (128 << 10)) step_waves /= 2;
    Shape shape{row_waves, step_waves, 0};
    const int threads = row_waves * step_waves * 64;
    while ((1 << shape.chunk_log2) < step_waves) ++shape.chunk_log2;
    const size_t sums = (size_t)step_waves * have * row_waves * 16 * NT * 4;
    const size_t x_bytes = WHOLE ? (size_t)steps * operand_units<X>(have) * 16
                                 : ((size_t)step_units<X>(G, T) * 16 << shape.chunk_log2) * ((1 << shape.chunk_log2) < steps ? 2 : 1);
    // (a launch takes 65535 workgroups the second way and fewer than 2^32 threads)
    const int64_t tiles = (1 << 27) / (steps * 16 * T), pass = 16 * T * (tiles < 1 ? 1 : (tiles < 32768 ? tiles : 32768));
    for (int64_t x0 = 0; x0 < a.tokens; x0 += pass) {
        Matvec4Args p = a;
        p.x = (const char*)a.x + x0 * a.ld_x * sizeof(X);
        p.y = (char*)a.y + x0 * a.ld_y * (a.y_type == LBFGSB_F32 ? 4 : sizeof(X));
        p.tokens = a.tokens - x0 < pass ? a.tokens - x0 : pass;
        if (!WHOLE) {
            p.operands = (char*)a.operands + (size_t)(x0 / (16 * T)) * steps * step_units<X>(G, T) * 16;
            const int64_t blocks = (p.tokens * steps * 16 + 255) / 256;
            hipLaunchKernelGGL((k_operands4<X, G, T>), dim3((unsigned)blocks), dim3(256), 0, st, p);
        }
        hipLaunchKernelGGL((k_matvec4<X, S, G, NT, T, WHOLE>), dim3((unsigned)((units + row_waves - 1) / row_waves), (unsigned)((p.tokens + 16 * T - 1) / (16 * T))),
                           dim3(threads), x_bytes > sums ? x_bytes : sums, st, p, shape);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Up to 16 rows of x are in LDS as a whole where they are no larger than this: two workgroups to a compute unit.
constexpr int64_t kWholeBytes = 80 << 10;
template <typename X>
int64_t whole_bytes(const Packed4& w, int64_t tokens) { return tokens * w.steps() * operand_units<X>(1) * 16; }

template <typename X, typename S, int G>
hipError_t matvec4(const Matvec4Args& a, hipStream_t st) {
    const int T = tiles_of(a.tokens, sizeof(X));
    const int64_t whole = T == 1 ? whole_bytes<X>(a.w, a.tokens) : 0;
    if (T == 1) {
        // More than one row of x is brought to LDS for two blocks of W at once, where that leaves a workgroup for every compute unit.  us, one / two:
        // 8 rows of bf16 x 65536 x 4096 41 / 32, 16 38.1 / 37.0, 5 of f16 x 50021 x 2600 21.3 / 19.9, 3 of f32 x 32768 x 2048 18.1 / 16.6, but one of
        // bf16 x 131072 x 4096 44.8 / 45.5 and 4 x 16384 x 4096 12.4 / 13.7, which eight waves take in 11.2.
        // The steps of many blocks are shared by eight waves where a row of x takes more than half of its room, which leaves two workgroups a compute unit, else by
        // four, of which there are four.  us, four / eight waves: one row of bf16 x 131072 x 4096 44 / 49, x 20600 208 / 209, x 30000 302 / 293, x 40900 409 / 396, of f32 x
        // 131072 x 6900 90 / 97, x 32800 x 13000 71 / 60.
        const bool many = a.w.blocks() >= 512;
        const int beside = a.tokens > 1 && many ? 2 : 1, share = beside == 1 && (!many || whole > kWholeBytes / 2) ? 8 : 4;
        const bool wide = a.w.blocks() >= 256;
        constexpr int NT = G == 1 ? 2 : 4;
        if (whole <= kWholeBytes && wide) {
            if constexpr (sizeof(S) == 2)
                return a.w.scale_type == LBFGSB_BF16 ? matvec4_in<X, __bf16, G, NT, 1, true>(a, beside, share, st)
                                                     : matvec4_in<X, _Float16, G, NT, 1, true>(a, beside, share, st);
            else
                return matvec4_in<X, S, G, NT, 1, true>(a, beside, share, st);
        }
        if (whole <= kWholeBytes) return matvec4_in<X, S, G, 1, 1, true>(a, 1, 8, st);
        return wide ? matvec4_in<X, S, G, NT, 1, false>(a, beside, share, st) : matvec4_in<X, S, G, 1, 1, false>(a, 1, 8, st);
    }
    // Tiles of the weights to a wave: more of them read less of x, fewer leave more workgroups.  us for rows of W x 4096, groups of 128, one / two / four tiles:
    //            8192              16384             32768             65536
    // 32 bf16    19.4 / 26.0       20.5 / 26.7       27.2 / 29.1       48.0 / 38.7 / 43.8
    // 48 bf16    24.9 / 30.3       25.9 / 31.3       35.2 / 33.5       59.5 / 45.8 / 52.7
    // 64 bf16    26.9 / 37.6 / 54  28.3 / 38.5 / 55  39.1 / 41.5 / 56  68.0 / 74.1 / 60.7
    // 32 f32     31.0 / - / 57     32.6 / - / 57     57.3 / - / 59     107 / 78 / 66.8
    const bool large = a.w.blocks() >= 768;
    if (T == 2) return large ? matvec4_in<X, S, G, sizeof(X) == 2 || G == 1 ? 2 : 4, 2, false>(a, 4, 2, st) : matvec4_in<X, S, G, 1, 2, false>(a, 4, 2, st);
    if constexpr (sizeof(X) == 2) {
        if (T == 3) return a.w.blocks() >= 512 ? matvec4_in<X, S, G, 2, 3, false>(a, 4, 2, st) : matvec4_in<X, S, G, 1, 3, false>(a, 4, 2, st);
        return large ? matvec4_in<X, S, G, G == 4 ? 4 : 2, 4, false>(a, 4, 2, st) : matvec4_in<X, S, G, 1, 4, false>(a, 4, 2, st);
    }
    return hipErrorInvalidValue;
}

template <typename X, typename S>
hipError_t matvec4_by_group(const Matvec4Args& a, hipStream_t st) {
    const int g = depth_of(a.w.group_log2);
    return g == 1 ? matvec4<X, S, 1>(a, st) : (g == 2 ? matvec4<X, S, 2>(a, st) : matvec4<X, S, 4>(a, st));
}

}  // namespace

template <typename X>
size_t matvec4_space(const Packed4& w, int64_t tokens) {
    const int T = tiles_of(tokens, sizeof(X));
    if (T == 1 && whole_bytes<X>(w, tokens) <= kWholeBytes) return 0;
    return (size_t)((tokens + 16 * T - 1) / (16 * T)) * w.steps() * step_units<X>(depth_of(w.group_log2), T) * 16;
}

template <typename X>
hipError_t matvec4_of(const Matvec4Args& a, hipStream_t st) {
    return a.w.scale_type == LBFGSB_F32 ? matvec4_by_group<X, float>(a, st) : matvec4_by_group<X, uint16_t>(a, st);
}

}  // namespace lb
