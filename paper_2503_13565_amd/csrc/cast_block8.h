// The cast of one 32-element block to E4M3 by a quad of lanes (arXiv 2503.13565, section 3.4.3 with the 8-bit element format), shared by
// the cast of whole tensors (e4m3.hip) and the norm that leaves its rows in 8 bits (norm.hip).
#pragma once

#include "common.h"

namespace mxfp4 {

typedef __attribute__((ext_vector_type(2))) short s16x2_t;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2_t;

// Code (eeeemmm) of one element from its 15 magnitude bits and the block's scale byte.  With sig
// the 8-bit significand, r = |v| / X = sig * 2^(e - 7), e = exponent field - scale byte.  F is r in
// units of 2^-17; the quantum of E4M3 is 2^-9 below 2^-6 and 2^(binade - 3) above; F is rounded to
// it to nearest even and re-based to the code, saturating at 126 (448).
__device__ __forceinline__ uint32_t quantise_e4m3(uint32_t mag, int scale_byte)
{
    const uint32_t exp = mag >> 7;
    const uint32_t man = mag & 0x7Fu;
    const uint32_t sig = exp ? (0x80u | man) : man;
    const int sh = (int)(exp ? exp : 1u) - scale_byte + 10;
    if (sh < 0 || sig == 0u)
        return 0u;                                   // below 2^-10: rounds to zero
    const uint32_t F = sig << sh;                    // sh <= 18: below 2^26
    const int top = 31 - __clz((int)F);
    const int shq = (top > 11 ? top : 11) - 3;       // log2 of the quantum in F units
    const uint32_t rounded = (F + ((1u << (shq - 1)) - 1u) + ((F >> shq) & 1u)) >> shq;
    const uint32_t code = rounded + ((uint32_t)(shq - 8) << 3);
    return code > 126u ? 126u : code;
}

template <bool kHw>
__device__ __forceinline__ void cast_group8(const u32x4_t v, u32x2_t* out, int* scale_out)
{
    const uint32_t d[4] = {v[0], v[1], v[2], v[3]};
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        amax = max(amax, max(d[i] & 0x7FFFu, (d[i] >> 16) & 0x7FFFu));
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0xB1, 0xF, 0xF, false));
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4E, 0xF, 0xF, false));

    u32x2_t packed = {0u, 0u};
    int scale_byte;
    if (amax >= 0x7F80u) {
        scale_byte = 0xFF;                           // NaN or Inf in the block
    } else {
        scale_byte = (int)(amax >> 7) - 8;           // biased exponent of amax, minus 8
        scale_byte = scale_byte < 0 ? 0 : scale_byte;
        if constexpr (kHw) {
            const float scale = __uint_as_float((uint32_t)scale_byte << 23);
            const uint32_t top = (((uint32_t)scale_byte + 8u) << 7) | 0x60u;      // 448 X as BF16 magnitude bits
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = min(d[i] & 0x7FFFu, top) | (d[i] & 0x8000u);
                const uint32_t hi = min((d[i] >> 16) & 0x7FFFu, top) | ((d[i] >> 16) & 0x8000u);
                const uint32_t pair = lo | (hi << 16);
                s16x2_t r = {0, 0};
                r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, pair), scale, false);
                const uint32_t two = (uint32_t)(uint16_t)r[0];
                if (i < 2)
                    packed[0] |= two << (16 * i);
                else
                    packed[1] |= two << (16 * (i - 2));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = d[i] & 0xFFFFu, hi = d[i] >> 16;
                const uint32_t blo = quantise_e4m3(lo & 0x7FFFu, scale_byte) | ((lo >> 15) << 7);
                const uint32_t bhi = quantise_e4m3(hi & 0x7FFFu, scale_byte) | ((hi >> 15) << 7);
                const uint32_t two = blo | (bhi << 8);
                if (i < 2)
                    packed[0] |= two << (16 * i);
                else
                    packed[1] |= two << (16 * (i - 2));
            }
        }
    }
    *out = packed;
    *scale_out = scale_byte;
}

}  // namespace mxfp4
