// Launchers behind lsh_w4.h.  Arguments are already validated (w4_api.cpp);
// every launcher only enqueues work on `stream`.
#pragma once

#include "launch_cache.h"

namespace lsh {

// Packed weights: tiles of 16 outputs x 128 inputs, a row of tiles after the
// other.  A tile's codes are 64 x 16 bytes, piece l those of output l % 16: for
// i of 0 .. 3 a word with inputs 32 i + 8 (l / 16) .. + 7, the operand of lane l
// for one 16 x 16 x 32 product, so that a wave's load is 1 KB without gaps.
// Its INT4 scales and zero points are [4][per_tile][4], those of outputs 4 q ..
// + 3 next to each other (per_tile = 128 / group), its E2M1 scales [16][4].  Outputs past N and inputs past K hold codes of 0 and
// scales of 0.
struct W4Shape {
    int N, K, e2m1, group, zeros;
    int64_t tiles_n, tiles_k;  // ceil(N / 16), ceil(K / 128)
    __host__ __device__ int per_tile() const { return 128 / group; }
    __host__ __device__ size_t scale_bytes() const { return e2m1 ? 1 : 2; }
    __host__ __device__ size_t codes_size() const { return (size_t)(tiles_n * tiles_k) * 1024; }
    __host__ __device__ size_t scales_size() const {
        return ((size_t)(tiles_n * tiles_k) * 16 * per_tile() * scale_bytes() + 255) & ~(size_t)255;
    }
    __host__ __device__ size_t zeros_size() const {
        return zeros ? ((size_t)(tiles_n * tiles_k) * 16 * per_tile() + 255) & ~(size_t)255 : 0;
    }
    size_t bytes() const { return codes_size() + scales_size() + zeros_size(); }
};

// What lane `lane` of a wave reads of `a` to fill its LDS copies with, in bytes from
// the first row of the workgroup's tile (TM rows) on, 256 k for tile k of 128 inputs
// on top: the wave's copies are runs `run` + j of eight rows of one half (64 inputs),
// 16 bytes a lane.  `after` rows follow the tile's first.  Rows past the last
// one repeat it, and pieces past the end of a row its first piece of the tile (neither
// is used), so that every byte read is a byte of the matrix and nothing rests on how a
// buffer's bound counts a scalar offset (1% of a long call's time: 2048 x 4096 x 1024
// with the offsets in scalar registers 25.5 us, so 25.7).
template <int TM, int COPIES>
struct W4RowCopies {
    uint32_t at[COPIES], col;
    __host__ __device__ W4RowCopies(int lane, int run, int64_t after, uint32_t row_bytes) {
        // lane l fills slot l % 8 of row l / 8; piece p of row r is in slot p ^ (r & 7)
        col = 128u * (run / (TM / 8)) + 16u * ((lane & 7) ^ (lane >> 3));
        const int last = after < TM ? (int)after : TM - 1;
        for (int j = 0; j < COPIES; ++j) {
            const int row = 8 * (run % (TM / 8) + j) + (lane >> 3);
            at[j] = (uint32_t)(row < last ? row : last) * row_bytes + col;
        }
    }
    // Before the last tile, where it has `rest` bytes of each row's inputs (of 256).
    __host__ __device__ void shorten(uint32_t rest) {
        if (col < rest) return;
        for (int j = 0; j < COPIES; ++j) at[j] -= col;
    }
};

struct W4Call {
    int64_t M, a_stride;
    const uint16_t* a;
    const char* packed;
    const float *bias, *resid;
    float sign;
    int relu;
    float* out_f32;
    uint16_t* out_bf16;
};

hipError_t launch_w4_quantize(const W4Shape& s, bool f32, const void* w, char* packed, hipStream_t stream);
hipError_t launch_w4_pack(const W4Shape& s, const uint8_t* codes, const void* scales, const uint8_t* zeros,
                          char* packed, hipStream_t stream);
hipError_t launch_w4_unpack(const W4Shape& s, bool f32, const char* packed, void* w, hipStream_t stream);

size_t w4_workspace_bytes(const W4Shape& s, int64_t M);
hipError_t launch_linear_w4(const W4Shape& s, const W4Call& c, void* workspace, hipStream_t stream);

}  // namespace lsh
