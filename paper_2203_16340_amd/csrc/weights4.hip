// Weights of 4 bits: quantising a matrix, laying codes out for the products (matvec4.h), and the products' types.
#include "weights4.h"

namespace lb {

namespace {

typedef unsigned int u4 __attribute__((ext_vector_type(4)));

template <typename F>
hipError_t by_type(int dtype, F f) {
    return dtype == LBFGSB_F32 ? f(float{}) : (dtype == LBFGSB_BF16 ? f(__bf16{}) : f(_Float16{}));
}

// A thread for each 16 bytes that a lane loads, gathered byte by byte from a row, which is what bounds it: 131072 x 4096 takes 1.02 ms with its scales' launch, 4096 x 2048
// 18 us, where the bytes, read and written once, are 95 us and 1.5.  Once for weights that are multiplied many times over, so tiles through LDS were not tried.
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

// A wave a group, which it reads twice, the second time out of the caches, one or two entries a lane at a time, which bounds it: 131072 x 4096 bf16 takes 1.57 ms, 4096 x 2048 28 us,
// 32768 x 2048 f32 205 us, where the bytes are 227 us, 3.5 and 51.  Once for weights that are multiplied many times over, as above.
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

size_t matvec4_bytes(const Packed4& w, int64_t tokens, int x_type) {
    size_t n = 0;
    by_type(x_type, [&](auto x) { return n = matvec4_space<decltype(x)>(w, tokens), hipSuccess; });
    return (n + 255) & ~(size_t)255;
}

hipError_t launch_matvec4(const Matvec4Args& a, int x_type, hipStream_t st) {
    if (a.tokens == 0) return hipSuccess;
    return by_type(x_type, [&](auto x) { return matvec4_of<decltype(x)>(a, st); });
}

}  // namespace lb
