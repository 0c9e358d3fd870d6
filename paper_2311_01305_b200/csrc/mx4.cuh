// Shared pieces of the microscaled 4-bit operators: elements e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), two to a
// byte, the even column in the low half; one 8-bit scale for each block of a row's columns.
//   AWEQ_MX4_E8M0  blocks of 32, scale 2^(byte - 127)
//   AWEQ_MX4_E4M3  blocks of 16, scale e4m3, and a binary32 step per row
// The scales lie as the tensor cores take them: tiles of 128 rows x 4 blocks (512 bytes), the four scales of a row together,
// rows r, r + 32, r + 64, r + 96 side by side; tiles along the columns first, whole groups of 256 columns.
#pragma once
#include "common.cuh"
#include "kernels.h"

namespace aweq {

constexpr int kMx4Tile = 512;
__host__ __device__ constexpr int mx4_block(int fmt) { return fmt == AWEQ_MX4_E8M0 ? 32 : 16; }
// tiles of a 128-row block for 256 columns, and for all of them
__host__ __device__ constexpr int mx4_group_tiles(int fmt) { return fmt == AWEQ_MX4_E8M0 ? 2 : 4; }
__host__ __device__ inline long long mx4_row_tiles(long long cols, int fmt) { return (cols + 255) / 256 * mx4_group_tiles(fmt); }
__device__ __forceinline__ long long mx4_scale_at(long long row, int block, long long row_tiles)
{
    return ((row >> 7) * row_tiles + (block >> 2)) * kMx4Tile + (row & 31) * 16 + (row >> 5 & 3) * 4 + (block & 3);
}

struct Mx4LinearArgs {
    const unsigned char *X, *W, *x_scales, *w_scales;
    const float *x_step, *w_step, *bias;       // steps of rows: E4M3 only
    long long N, ldo;
    int K, O, fmt;
    uint16_t *out;
    aweq_dev_status *st;
};

}  // namespace aweq
