// Products with weights of 4 bits: the layouts, arguments and launches.
#pragma once

#include "logits.h"

namespace lb {

// How the codes lie where they are multiplied.  Rows go in blocks of 64, columns in steps of 128; of a block and step there are 4 tiles of
// 16 rows, tile t holding rows 4 c + t (c = 0 .. 15).  A lane's 16 bytes of a tile are what it feeds to four matrix instructions of
// depth 32: lane l has row c = l % 16 and, in word j, columns 32 j + 8 (l / 16) .. + 7, the code of column i in the low half of
// byte i, that of column 4 + i in the high one.  So a tile is one load of 1024 bytes by a wave, a group of 32 is whole in one
// instruction, and a lane's scales of the four tiles stand side by side.
// Behind the codes, for each block and group: 64 scales, and 64 zeros if there are any.  Rows and columns past the end have code and scale 0.
constexpr int kBlockRows = 64, kStepCols = 128, kStepBytes = kBlockRows * kStepCols / 2, kTileBytes = kStepBytes / 4;

struct Packed4 {
    int64_t rows;
    int cols, group_log2, scale_type, zeros;
    __host__ __device__ int64_t blocks() const { return (rows + kBlockRows - 1) / kBlockRows; }
    __host__ __device__ int steps() const { return (cols + kStepCols - 1) / kStepCols; }
    __host__ __device__ int groups() const { return (int)(((int64_t)cols + (1ll << group_log2) - 1) >> group_log2); }
    __host__ __device__ size_t code_bytes() const { return (size_t)blocks() * steps() * kStepBytes; }
    size_t bytes() const { return code_bytes() + (size_t)blocks() * groups() * kBlockRows * (1 + zeros) * (scale_type == LBFGSB_F32 ? 4 : 2); }
};

struct Matvec4Args {
    Packed4 w;
    const void* packed;
    int64_t tokens, ld_x, ld_y;
    const void* x;
    void* y;
    int y_type;
    void* operands;              // workspace: x as operands (more than 16 tokens)
};

// tiles of 16 rows of x that are multiplied in one pass over the weights
inline int tiles_of(int64_t tokens, size_t size_x) { return tokens <= 16 ? 1 : (tokens <= 32 || size_x == 4 ? 2 : (tokens <= 48 ? 3 : 4)); }
// matrix instructions between two groups
inline int depth_of(int group_log2) { return group_log2 == 5 ? 1 : (group_log2 == 6 ? 2 : 4); }

hipError_t launch_quantize4(int dtype, int64_t ld, const void* w, int64_t rows, int64_t cols, int64_t group, int scale_type, uint8_t* codes, void* scale,
                            void* zero, hipStream_t st);
hipError_t launch_pack4(const Packed4& w, const uint8_t* codes, const void* scale, const void* zero, void* packed, hipStream_t st);
hipError_t launch_matvec4(const Matvec4Args& a, int x_type, hipStream_t st);
size_t matvec4_bytes(const Packed4& w, int64_t tokens, int x_type);     // of workspace
// the same for one type of x, tokens > 0 (matvec4.h)
template <typename X>
hipError_t matvec4_of(const Matvec4Args& a, hipStream_t st);
template <typename X>
size_t matvec4_space(const Packed4& w, int64_t tokens);

}  // namespace lb
