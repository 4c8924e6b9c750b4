// Device helpers of the grouped products, the products in 8-bit integers and the AdamW step.
#pragma once

#include "groot_device.h"
#include "groot_dense_ops.h"

namespace groot {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// Group and rows of one tile of kRows rows: tiles are numbered group after group, every group begins a new one.  The whole
// wavefront looks at 64 groups at a time.  An offset outside [0, n] is taken as the nearer end.
struct RowTile {
    int32_t group;                           // -1: there is no such tile
    int64_t begin, end;                      // rows of the tile
};

// a value that is the same in every lane, as a scalar
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

template <int kRows>
__device__ __forceinline__ RowTile find_tile(const int64_t *__restrict__ offsets, int32_t groups, int64_t n, int64_t tile)
{
    if (!offsets) {
        const int64_t begin = tile * kRows;
        return RowTile{begin < n ? 0 : -1, begin, begin + kRows < n ? begin + kRows : n};
    }
    const int lane = threadIdx.x % kWave;
    int64_t before = 0;
    for (int32_t g0 = 0; g0 < groups; g0 += kWave) {
        const int32_t g = g0 + lane;
        int64_t b = 0, e = 0;
        if (g < groups) {
            b = offsets[g];
            e = offsets[g + 1];
            b = b < 0 ? 0 : b > n ? n : b;
            e = e < b ? b : e > n ? n : e;
        }
        int64_t upto = (e - b + kRows - 1) / kRows;      // tiles of this and the groups before it
        const int64_t mine = upto;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int64_t o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const int64_t all = __shfl(upto, kWave - 1);
        if (tile < before + all) {
            const int at = __popcll(__ballot(before + upto <= tile));
            const int64_t first = before + __shfl(upto, at) - __shfl(mine, at);
            const int64_t gb = __shfl(b, at), ge = uniform(__shfl(e, at)), begin = uniform(gb + (tile - first) * kRows);
            return RowTile{__builtin_amdgcn_readfirstlane(g0 + at), begin, begin + kRows < ge ? begin + kRows : ge};
        }
        before += all;
    }
    return RowTile{-1, 0, 0};
}

__device__ __forceinline__ void group_rows(const int64_t *__restrict__ offsets, int64_t n, int32_t g, int64_t *begin, int64_t *end)
{
    int64_t b = 0, e = n;
    if (offsets) {
        b = offsets[g];
        e = offsets[g + 1];
        b = b < 0 ? 0 : b > n ? n : b;
        e = e < b ? b : e > n ? n : e;
    }
    *begin = b;
    *end = e;
}

}  // namespace groot
