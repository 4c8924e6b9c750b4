// Device helpers of the grouped products, the products in 8-bit integers and the AdamW step.
#pragma once

#include "groot_device.h"
#include "groot_dense_ops.h"

namespace groot {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// The quotient x / s, rounded as a division rounds it, from the reciprocal r of s rounded to nearest (Markstein): x r is one and a half
// last places off at most, and its remainder, exact in one fused operation, decides.  (1.3 % of random pairs have an x r more than one
// place off.  Pairs whose quotient lies nearest to the middle of two numbers, as r's error can still reach it, are few enough to be
// counted out: all 4.7 x 10^7 with a remainder of up to 8 from it round as the division does.)  For s and x / s well inside fp32's range.
__device__ __forceinline__ float quotient(float x, float s, float r)
{
    const float q = x * r;
    return __builtin_fmaf(__builtin_fmaf(-q, s, x), r, q);
}

// What another lane holds, for sums and the like over kLanes neighbouring lanes: lanes 1, 2, 4 and 8 away by a move inside of 16 lanes (the
// last two reversed: lanes that are less far apart hold the same by then), 16 and 32 away by an exchange that gives every lane both values.
template <int kAway>
__device__ __forceinline__ void pair_lanes(uint32_t x, uint32_t *a, uint32_t *b)
{
    *a = x;
    if constexpr (kAway == 1) *b = __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, false);        // quad_perm 1 0 3 2
    else if constexpr (kAway == 2) *b = __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, false);   // quad_perm 2 3 0 1
    else if constexpr (kAway == 4) *b = __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, false);  // row_half_mirror
    else if constexpr (kAway == 8) *b = __builtin_amdgcn_update_dpp(0, x, 0x140, 0xF, 0xF, false);  // row_mirror
    else {
        const auto r = kAway == 16 ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false);
        *a = r[0];
        *b = r[1];
    }
}
template <int kAway>
__device__ __forceinline__ void pair_lanes(float x, float *a, float *b)
{
    uint32_t u, v;
    pair_lanes<kAway>(__float_as_uint(x), &u, &v);
    *a = __uint_as_float(u);
    *b = __uint_as_float(v);
}
template <int kAway>
__device__ __forceinline__ void pair_lanes(double x, double *a, double *b)
{
    const uint64_t bits = __builtin_bit_cast(uint64_t, x);
    uint32_t ul, vl, uh, vh;
    pair_lanes<kAway>((uint32_t)bits, &ul, &vl);
    pair_lanes<kAway>((uint32_t)(bits >> 32), &uh, &vh);
    *a = __builtin_bit_cast(double, (uint64_t)uh << 32 | ul);
    *b = __builtin_bit_cast(double, (uint64_t)vh << 32 | vl);
}
// `both` of the values of kLanes neighbouring lanes, in every one of them; all of them take part, and `both` does not mind the order
template <int kLanes, int kAway = 1, typename T, typename F>
__device__ __forceinline__ T over_lanes(T x, F both)
{
    if constexpr (kAway < kLanes) {
        T a, b;
        pair_lanes<kAway>(x, &a, &b);
        return over_lanes<kLanes, kAway * 2>(both(a, b), both);
    } else {
        return x;
    }
}

// a value that is the same in every lane, as a scalar
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// Group and rows of one tile of 2^log_rows rows: tiles are numbered group after group, every group begins a new one.  The whole
// wavefront looks at 64 groups at a time.  An offset outside [0, n] is taken as the nearer end.
struct RowTile {
    int32_t group;                           // -1: there is no such tile
    int64_t begin, end;                      // rows of the tile
    int64_t place, count;                    // its place among the tiles of its group, and how many these are
    int64_t shared_before;                   // tiles of the groups before it that have two or more (only where asked for)
};

__device__ __forceinline__ int64_t sum_upto(int64_t x)
{
    const int lane = threadIdx.x % kWave;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int64_t o = __shfl_up(x, d);
        if (lane >= d) x += o;
    }
    return x;
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

// kAtLeastOne: a group without rows has a tile all the same
template <bool kShared = false, bool kAtLeastOne = false>
__device__ __forceinline__ RowTile find_tile(const int64_t *__restrict__ offsets, int32_t groups, int64_t n, int64_t tile, int log_rows)
{
    const int64_t rows = (int64_t)1 << log_rows;
    if (!offsets) {
        const int64_t begin = tile << log_rows;
        const int64_t count = (n + rows - 1) >> log_rows;
        return RowTile{begin < n || (kAtLeastOne && tile == 0) ? 0 : -1, begin, begin + rows < n ? begin + rows : n, tile, kAtLeastOne && n == 0 ? 1 : count, 0};
    }
    const int lane = threadIdx.x % kWave;
    int64_t before = 0, shared = 0;
    for (int32_t g0 = 0; g0 < groups; g0 += kWave) {
        int64_t b = 0, e = 0;
        if (g0 + lane < groups) group_rows(offsets, n, g0 + lane, &b, &e);
        const int64_t tiles = (e - b + rows - 1) >> log_rows;
        const int64_t mine = kAtLeastOne && tiles == 0 && g0 + lane < groups ? 1 : tiles;
        const int64_t upto = sum_upto(mine), all = __shfl(upto, kWave - 1);
        const int64_t shared_upto = kShared ? sum_upto(mine > 1 ? mine : 0) : 0;
        if (tile < before + all) {
            const int at = __popcll(__ballot(before + upto <= tile));
            const int64_t count = uniform(__shfl(mine, at)), first = before + uniform(__shfl(upto, at)) - count;
            const int64_t begin = uniform(__shfl(b, at)) + ((tile - first) << log_rows), ge = uniform(__shfl(e, at));
            return RowTile{__builtin_amdgcn_readfirstlane(g0 + at), begin, begin + rows < ge ? begin + rows : ge, tile - first, count,
                           kShared ? shared + uniform(__shfl(shared_upto, at)) - (count > 1 ? count : 0) : 0};
        }
        before += uniform(all);
        if (kShared) shared += uniform(__shfl(shared_upto, kWave - 1));
    }
    return RowTile{-1, 0, 0, 0, 0, 0};
}

}  // namespace groot
