// Weights of 4 bits: quantising a matrix, laying codes out for the products, and the products y = x W^T of a few rows x.
//
// With w = scale (code - zero) a group's part of a product is scale (sum_j code_j x_j - zero sum_j x_j).  Codes are whole numbers of 4 bits, exact in
// bf16 and f16, so the two sums are matrix instructions on the codes themselves and on ones, with exact products and sums in 32 bits; scale and zero
// enter once a group.  x in 32 bits goes in as three bf16 parts, which hold its 24 bits.
//
// Bound by memory: half a byte and one or two instructions a weight.  A code becomes a matrix operand in 7/8 of an instruction: a byte
// 0 .. 15 is, read as an 8-bit float with 3 bits of mantissa, that number times 2^-9 (denormal below 8, the first binade from there), so masking
// the two halves of a word and four conversions of pairs with a scale of 2^9 make eight of them.
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

template <typename S>
struct Scales {
    typedef S four __attribute__((ext_vector_type(4)));
};

// A wave's share of 16 rows of x against NT tiles of a block: steps wave, wave + waves, ...  The waves' sums are joined in LDS in a fixed order.
// x's row i stands at row 4 (i % 4) + i / 4 of the operand, so that up to four rows take one of the four result registers.
template <typename X, typename S, int G, int NT>    // G: matrix instructions between two groups, 1, 2 or 4
__global__ __launch_bounds__(512) void k_matvec4(Matvec4Args a) {
    extern __shared__ float lds[];
    typedef typename OperandOf<X>::type M;
    typedef typename Operand<M>::vec vec;
    typedef typename Scales<S>::four S4;
    constexpr int kRows = 16 * NT;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int c = lane & 15, kq = lane >> 4;
    const int64_t block = blockIdx.x / (4 / NT);
    const int tile = (int)(blockIdx.x % (4 / NT)) * NT;
    const int64_t x0 = (int64_t)blockIdx.y * 16;
    const int have = (int)(a.tokens - x0 < 16 ? a.tokens - x0 : 16);
    const int mine = 4 * (c & 3) + (c >> 2);           // the row of x whose entries this lane loads
    const bool live = mine < have;
    const X* xr = (const X*)a.x + (x0 + (live ? mine : 0)) * a.ld_x + kq * 8;
    const int steps = a.w.steps(), cols = a.w.cols, groups = a.w.groups();
    const char* codes = (const char*)a.packed + (size_t)block * steps * kStepBytes + tile * kTileBytes + lane * 16;
    const S* scales = (const S*)((const char*)a.packed + a.w.code_bytes()) + (size_t)block * groups * kBlockRows * (1 + a.w.zeros) + 4 * c + tile;
    const int each = kBlockRows * (1 + a.w.zeros);

    f4 y[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) y[t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    vec ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (M)1.0f;

    struct Step {
        u4 w[NT];
        X x[4][8];
        float scale[4 / G][NT], zero[4 / G][NT];
    };
    auto load = [&](Step& st, int s) {
#pragma unroll
        for (int t = 0; t < NT; ++t) st.w[t] = __builtin_nontemporal_load((const u4*)(codes + (size_t)s * kStepBytes + t * kTileBytes));
        if (live && (s + 1) * kStepCols <= cols) {
            typedef X wide __attribute__((ext_vector_type(8), aligned(sizeof(X))));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const wide v = *(const wide*)(xr + s * kStepCols + j * 32);
#pragma unroll
                for (int e = 0; e < 8; ++e) st.x[j][e] = v[e];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int k = s * kStepCols + j * 32 + e;
                    st.x[j][e] = live && k + kq * 8 < cols ? xr[k] : (X)0.0f;
                }
        }
#pragma unroll
        for (int g = 0; g < 4 / G; ++g) {
            // (a last group may end before its step does; what comes after it is 0 times the scale of a group that is there)
            const int at = min((s * kStepCols + g * G * 32) >> a.w.group_log2, groups - 1);
            const S* from = scales + (size_t)at * each;
            if constexpr (NT == 4) {
                const S4 v = *(const S4*)from;
#pragma unroll
                for (int t = 0; t < NT; ++t) st.scale[g][t] = (float)v[t];
                if (a.w.zeros) {
                    const S4 z = *(const S4*)(from + kBlockRows);
#pragma unroll
                    for (int t = 0; t < NT; ++t) st.zero[g][t] = (float)z[t];
                }
            } else {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    st.scale[g][t] = (float)from[t];
                    if (a.w.zeros) st.zero[g][t] = (float)from[kBlockRows + t];
                }
            }
        }
        if (!a.w.zeros)
#pragma unroll
            for (int g = 0; g < 4 / G; ++g)
#pragma unroll
                for (int t = 0; t < NT; ++t) st.zero[g][t] = 8.0f;
    };
    auto multiply = [&](const Step& st) {
        f4 sum[NT], all;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            Parts<X> x;
            x.set(st.x[j]);
            if (j % G == 0) {
                all = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
            }
#pragma unroll
            for (int n = 0; n < Parts<X>::N; ++n) all = Operand<M>::product(x.p[n], ones, all);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const vec w = unpacked<M>(st.w[t][j]);
#pragma unroll
                for (int n = 0; n < Parts<X>::N; ++n) sum[t] = Operand<M>::product(x.p[n], w, sum[t]);
            }
            if (j % G == G - 1) {
                const int g = j / G;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (r == 0 || have > 4) y[t][r] = fmaf(st.scale[g][t], fmaf(-st.zero[g][t], all[r], sum[t][r]), y[t][r]);
            }
        }
    };
    Step now, next;
    if (wave < steps) load(next, wave);
    for (int s = wave; s < steps; s += waves) {
        now = next;
        if (s + waves < steps) load(next, s + waves);
        multiply(now);
    }

    // register r holds row 4 r + kq of x
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int i = 4 * r + kq;
        if (i < have) {
#pragma unroll
            for (int t = 0; t < NT; ++t) lds[(wave * have + i) * kRows + (NT == 4 ? 4 * c + t : c)] = y[t][r];
        }
    }
    __syncthreads();
    for (int k = threadIdx.x; k < have * kRows; k += blockDim.x) {
        const int i = k / kRows, o = k % kRows;
        const int64_t row = block * kBlockRows + (NT == 4 ? o : 4 * o + tile);
        float sum = 0.0f;
        for (int w = 0; w < waves; ++w) sum += lds[w * have * kRows + k];
        if (row < a.w.rows) {
            const int64_t at = (x0 + i) * a.ld_y + row;
            if (a.y_type == LBFGSB_F32) ((float*)a.y)[at] = sum;
            else ((X*)a.y)[at] = (X)sum;
        }
    }
}

template <typename X, typename S, int G>
hipError_t matvec4(const Matvec4Args& a, hipStream_t st) {
    const int64_t blocks = a.w.blocks();
    const int waves = a.w.steps() < 8 ? a.w.steps() : 8;
    const int have = a.tokens < 16 ? (int)a.tokens : 16;
    for (int64_t x0 = 0; x0 < a.tokens; x0 += 16 * 32768) {
        Matvec4Args p = a;
        const size_t bx = sizeof(X), by = a.y_type == LBFGSB_F32 ? 4 : sizeof(X);
        p.x = (const char*)a.x + x0 * a.ld_x * bx;
        p.y = (char*)a.y + x0 * a.ld_y * by;
        p.tokens = a.tokens - x0 < 16 * 32768 ? a.tokens - x0 : 16 * 32768;
        const unsigned tiles = (unsigned)((p.tokens + 15) / 16);
        if (blocks >= 256)
            hipLaunchKernelGGL((k_matvec4<X, S, G, 4>), dim3((unsigned)blocks, tiles), dim3(waves * 64), (size_t)waves * have * 64 * 4, st, p);
        else
            hipLaunchKernelGGL((k_matvec4<X, S, G, 1>), dim3((unsigned)(blocks * 4), tiles), dim3(waves * 64), (size_t)waves * have * 16 * 4, st, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename X, typename S>
hipError_t matvec4_by_group(const Matvec4Args& a, hipStream_t st) {
    return a.w.group_log2 == 5 ? matvec4<X, S, 1>(a, st) : (a.w.group_log2 == 6 ? matvec4<X, S, 2>(a, st) : matvec4<X, S, 4>(a, st));
}

template <typename F>
hipError_t by_type(int dtype, F f) {
    return dtype == LBFGSB_F32 ? f(float{}) : (dtype == LBFGSB_BF16 ? f(__bf16{}) : f(_Float16{}));
}

// A thread for each 16 bytes that a lane loads.
__global__ __launch_bounds__(256) void k_pack4(Packed4 w, const uint8_t* codes, u4* packed, int64_t pieces) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const int lane = (int)(i & 63), tile = (int)(i >> 6) & 3, steps = w.steps();
    const int64_t at = i >> 8, block = at / steps;
    const int step = (int)(at - block * steps);
    const int64_t row = block * kBlockRows + 4 * (lane & 15) + tile, wide = ((int64_t)w.cols + 1) / 2;
    u4 out = {0, 0, 0, 0};
    if (row < w.rows) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int col = step * kStepCols + 32 * j + 8 * (lane >> 4);
            unsigned word = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < w.cols) {
                    const unsigned code = (codes[row * wide + (col + e) / 2] >> (4 * (e & 1))) & 15u;
                    word |= code << (8 * (e & 3) + 4 * (e >> 2));
                }
            out[j] = word;
        }
    }
    packed[i] = out;
}
// S: as many bits as a scale has
template <typename S>
__global__ __launch_bounds__(256) void k_pack4_scales(Packed4 w, const S* scale, const S* zero, S* packed, int64_t entries) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= entries) return;
    const int groups = w.groups(), each = kBlockRows * (1 + w.zeros);
    const int64_t at = i / each, block = at / groups;
    const int g = (int)(at - block * groups), o = (int)(i - at * each);
    const int64_t row = block * kBlockRows + (o & (kBlockRows - 1));
    packed[i] = row < w.rows ? (o < kBlockRows ? scale : zero)[row * groups + g] : (S)0;
}

// A wave a group.
template <typename T, typename S>
__global__ __launch_bounds__(256) void k_quantize4(int64_t ld, const T* w, int64_t rows, int64_t cols, int group_log2, uint8_t* codes, S* scale, S* zero) {
    const int64_t groups = (cols + (1ll << group_log2) - 1) >> group_log2, wide = (cols + 1) / 2;
    const int lane = threadIdx.x & 63;
    for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < rows * groups; i += (int64_t)gridDim.x * 4) {
        const int64_t r = i / groups, g = i - r * groups, from = g << group_log2, to = min(from + (1ll << group_log2), cols);
        const T* row = w + r * ld;
        float low = 0.0f, high = 0.0f;
        bool lost = false;
        for (int64_t k = from + lane; k < to; k += 64) {
            const float v = (float)row[k];
            lost |= !(fabsf(v) < INFINITY);
            low = fminf(low, v);
            high = fmaxf(high, v);
        }
        low = -wave_max_f(-low);
        high = wave_max_f(high);
        // (in 64 bits: the middle between two zeros is met exactly by rows as far below 0 as above it.  A spread past the end of a scale's type makes it infinite)
        S sc = (S)(float)(zero ? ((double)high - (double)low) / 15.0 : (double)fmaxf(high, -low) / 7.0);
        if (__any(lost)) sc = (S)NAN;
        const float step = (float)sc;
        const float offset = !zero ? 8.0f : (step > 0.0f ? (float)fmin(fmax(rint(-(double)low / (double)step), 0.0), 15.0) : 0.0f);
        auto code = [&](int64_t k) -> unsigned {
            if (k >= to) return 0;
            const float q = step > 0.0f ? rintf((float)row[k] / step) + offset : offset;
            return (unsigned)fminf(fmaxf(q, 0.0f), 15.0f);
        };
        for (int64_t k = from + 2 * lane; k < to; k += 128) codes[r * wide + k / 2] = (uint8_t)(code(k) | code(k + 1) << 4);
        if (lane == 0) {
            scale[i] = sc;
            if (zero) zero[i] = (S)offset;
        }
    }
}

int log2_of(int64_t n) {
    int l = 0;
    while ((1ll << l) < n) ++l;
    return l;
}

}  // namespace

hipError_t launch_quantize4(int dtype, int64_t ld, const void* w, int64_t rows, int64_t cols, int64_t group, int scale_type, uint8_t* codes, void* scale,
                            void* zero, hipStream_t st) {
    const int64_t all = rows * ((cols + group - 1) / group), grid = (all + 3) / 4;
    return by_type(dtype, [&](auto t) {
        typedef decltype(t) T;
        return by_type(scale_type, [&](auto s) {
            typedef decltype(s) S;
            hipLaunchKernelGGL((k_quantize4<T, S>), dim3((unsigned)(grid < 65536 ? grid : 65536)), dim3(256), 0, st, ld, (const T*)w, rows, cols, log2_of(group),
                               codes, (S*)scale, (S*)zero);
            return hipGetLastError();
        });
    });
}

hipError_t launch_pack4(const Packed4& w, const uint8_t* codes, const void* scale, const void* zero, void* packed, hipStream_t st) {
    const int64_t pieces = (int64_t)(w.code_bytes() / 16), entries = (int64_t)w.blocks() * w.groups() * kBlockRows * (1 + w.zeros);
    hipLaunchKernelGGL(k_pack4, dim3((unsigned)((pieces + 255) / 256)), dim3(256), 0, st, w, codes, (u4*)packed, pieces);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    void* to = (char*)packed + w.code_bytes();
    const dim3 grid((unsigned)((entries + 255) / 256));
    if (w.scale_type == LBFGSB_F32)
        hipLaunchKernelGGL(k_pack4_scales<uint32_t>, grid, dim3(256), 0, st, w, (const uint32_t*)scale, (const uint32_t*)zero, (uint32_t*)to, entries);
    else
        hipLaunchKernelGGL(k_pack4_scales<uint16_t>, grid, dim3(256), 0, st, w, (const uint16_t*)scale, (const uint16_t*)zero, (uint16_t*)to, entries);
    return hipGetLastError();
}

hipError_t launch_matvec4(const Matvec4Args& a, int x_type, hipStream_t st) {
    if (a.tokens == 0) return hipSuccess;
    return by_type(x_type, [&](auto x) {
        return by_type(a.w.scale_type, [&](auto s) { return matvec4_by_group<decltype(x), decltype(s)>(a, st); });
    });
}

}  // namespace lb
