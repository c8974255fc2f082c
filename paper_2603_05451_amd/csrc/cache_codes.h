// Codes of the quantised cache as pairs of 16-bit numbers (gfx950's conversions).  They take the scale as a float whose exponent
// field is the scale byte: 2^(byte - 127), byte 0 included; a byte of 255 gives NaN.  They round to the element type: bf16 holds
// every value below 2^128 exactly, fp16 is as a conversion from fp32 would be; both are infinite beyond their range.
#pragma once
#include "common.h"

namespace attn {

__device__ __forceinline__ float cache_scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// e2m1 codes of byte SEL of w
template <int SEL>
__device__ __forceinline__ uint32_t e2m1_pair(bf16, uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}
template <int SEL>
__device__ __forceinline__ uint32_t e2m1_pair(f16, uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, SEL));
}
// e4m3 codes of the low or the high half of w
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3_pair(bf16, uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
}
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3_pair(f16, uint32_t w, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HIGH));
}

// 8 channels of element type E (vector E8)
template <typename E8, typename E>
__device__ __forceinline__ E8 cache_e2m1(E e, uint32_t w, float scale)
{
    return __builtin_bit_cast(E8, u32x4{e2m1_pair<0>(e, w, scale), e2m1_pair<1>(e, w, scale), e2m1_pair<2>(e, w, scale), e2m1_pair<3>(e, w, scale)});
}
template <typename E8, typename E>
__device__ __forceinline__ E8 cache_e4m3(E e, uint32_t w0, uint32_t w1, float scale)
{
    return __builtin_bit_cast(E8, u32x4{e4m3_pair<false>(e, w0, scale), e4m3_pair<true>(e, w0, scale),
                                        e4m3_pair<false>(e, w1, scale), e4m3_pair<true>(e, w1, scale)});
}

// Whether 16 bytes of codes under this scale byte may hold numbers that are infinite or NaN as element type E (4 * 2^126 and 256 * 2^120
// are 2^128, 4 * 2^14 and 256 * 2^8 are 2^16; e4m3 has a NaN of its own).
template <int BITS, typename E>
__device__ __forceinline__ bool cache_odd(E, const uint32_t (&w)[4], uint32_t byte)
{
    constexpr bool f16_ = std::is_same_v<E, f16>;
    constexpr uint32_t finite = BITS == 4 ? (f16_ ? 140 : 252) : (f16_ ? 134 : 246);        // the largest scale without
    bool odd = byte > finite;
    if constexpr (BITS == 8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= (((w[e] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
    }
    return odd;
}

}  // namespace attn
