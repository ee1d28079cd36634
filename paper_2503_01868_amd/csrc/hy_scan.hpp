// Sums over the lanes of a wave that move by DPP, in registers: six steps of one or two moves and an addition, where each of
// __shfl_up's is a trip through LDS (a scan of doubles 0.1 us instead of 0.4).
#pragma once
#include "hy_common.hpp"

namespace hy {

template <int CTRL, int ROWS, typename X>
__device__ __forceinline__ X moved(X x) {  // lanes without a source get zero bits
    static_assert(sizeof(X) == 4 || sizeof(X) == 8, "one word or two");
    if constexpr (sizeof(X) == 4) {
        return __builtin_bit_cast(X, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
    } else {
        const u32x2_t w = __builtin_bit_cast(u32x2_t, x);
        const u32x2_t r = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[0], CTRL, ROWS, 0xf, false),
                           (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[1], CTRL, ROWS, 0xf, false)};
        return __builtin_bit_cast(X, r);
    }
}

// The sum of a lane and all in front of it.  All lanes take part.
template <typename X>
__device__ __forceinline__ X wave_upto(X x) {
    x += moved<0x111, 0xf>(x);  // of 16 lanes: from 1, 2, 4, 8 in front
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    x += moved<0x142, 0xa>(x);  // the 16 in front, to the second and the fourth
    x += moved<0x143, 0xc>(x);  // the 32 in front
    return x;
}

// Of lane `l`, the same for all.
template <typename X>
__device__ __forceinline__ X of_lane(X x, int l) {
    if constexpr (sizeof(X) == 4) {
        return __builtin_bit_cast(X, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l));
    } else {
        const u32x2_t w = __builtin_bit_cast(u32x2_t, x);
        const u32x2_t r = {(uint32_t)__builtin_amdgcn_readlane((int)w[0], l), (uint32_t)__builtin_amdgcn_readlane((int)w[1], l)};
        return __builtin_bit_cast(X, r);
    }
}

// The same number, but what is computed from it is computed where it is used and not kept in registers from before a loop.
__device__ __forceinline__ int fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

}  // namespace hy
