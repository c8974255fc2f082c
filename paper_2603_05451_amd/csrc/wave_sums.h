// Sums over the lanes of a wave.
#pragma once
#include "common.h"

namespace attn {

// Inclusive prefix sums over the lanes of a wave: within 16 lanes, then the ends of rows 0 and 2 to rows 1 and 3, then that of row 1 to
// both upper rows.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_moved(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int wave_prefix(int x)
{
    x = add_moved<0x111, 0xf>(x);          // row_shr 1, 2, 4, 8
    x = add_moved<0x112, 0xf>(x);
    x = add_moved<0x114, 0xf>(x);
    x = add_moved<0x118, 0xf>(x);
    x = add_moved<0x142, 0xa>(x);          // row_bcast 15
    return add_moved<0x143, 0xc>(x);       // row_bcast 31
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_prefix(x), 63); }
template <int CTRL, int ROWS>
__device__ __forceinline__ float add_moved(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_sum(float x)      // the same order of additions in every wave
{
    x = add_moved<0x111, 0xf>(x);
    x = add_moved<0x112, 0xf>(x);
    x = add_moved<0x114, 0xf>(x);
    x = add_moved<0x118, 0xf>(x);
    x = add_moved<0x142, 0xa>(x);
    x = add_moved<0x143, 0xc>(x);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

}  // namespace attn
