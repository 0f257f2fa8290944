// Sums over a wave's lanes up to each lane's own.
#pragma once

#include <hip/hip_runtime.h>

namespace ress {

// The value of the lane that CTRL names, 0 where there is none or ROWS (four lanes' rows of 16) leaves it out.
template <int CTRL, int ROWS>
__device__ __forceinline__ int lane_below(int x)
{
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}

// (By the vector unit's own moves: 1, 2, 4 and 8 lanes within 16, then the last lane of 16, and of 32, to those behind it. Through
// the LDS, as __shfl_up, each step takes its latency.) join(a, b): a sum of two, with join(x, 0) = x.
template <typename F>
__device__ __forceinline__ int scan_wave(int x, F join)
{
    x = join(x, lane_below<0x111, 0xf>(x));
    x = join(x, lane_below<0x112, 0xf>(x));
    x = join(x, lane_below<0x114, 0xf>(x));
    x = join(x, lane_below<0x118, 0xf>(x));
    x = join(x, lane_below<0x142, 0xa>(x));
    return join(x, lane_below<0x143, 0xc>(x));
}

// The sum of all lanes, the same in each.
__device__ __forceinline__ float sum_wave(float x)
{
    const int s = scan_wave(__builtin_bit_cast(int, x), [](int a, int b) {
        return __builtin_bit_cast(int, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
    });
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(s, 63));
}

}  // namespace ress
