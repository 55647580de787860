// The cast of one 32-element block to MXFP4 by a quad of lanes (arXiv 2503.13565, section 3.4.3), shared by the cast of
// whole tensors (cast.hip) and the store into a paged cache (kv_store.hip).
#pragma once

#include "common.h"

namespace mxfp4 {

// Code (eem) of one element from its 15 magnitude bits and the block's scale byte.
// With sig the 8-bit significand and d = exponent - scale byte (d <= 2 for every element of
// the block that produced the scale), F = |v|/X in units of 2^-10 is sig << (d+3).  The
// quantum of E2M1 is 0.5 below 2 and doubles per binade above; F is rounded to it to nearest
// even and the result is re-based to the code, saturating at 7.
__device__ __forceinline__ uint32_t quantise_e2m1(uint32_t mag, int scale_byte)
{
    const uint32_t exp = mag >> 7;
    const uint32_t man = mag & 0x7Fu;
    const uint32_t sig = exp ? (0x80u | man) : man;
    const int sh3 = (int)(exp ? exp : 1u) - scale_byte + 3;
    if (sh3 < 0)
        return 0u;                                   // below 2^-3 of X: rounds to zero
    const uint32_t F = sig << sh3;
    const int top = 31 - __clz((int)F);              // -1 for F == 0
    const int shq = (top > 10 ? top : 10) - 1;       // log2 of the quantum in F units
    const uint32_t rounded = (F + ((1u << (shq - 1)) - 1u) + ((F >> shq) & 1u)) >> shq;
    const uint32_t code = rounded + 2u * (uint32_t)(shq - 9);
    return code > 7u ? 7u : code;
}

// One 8-element group (16 bytes of BF16) of a block per lane; the four lanes of a quad hold one
// 32-element block.  kHw: elements are rounded by the gfx950 scaled BF16->FP4 convert (one
// instruction per element pair; checked on the device against the integer rule above for every
// finite BF16 value and every scale byte); otherwise by the integer rule.
template <bool kHw>
__device__ __forceinline__ void cast_group(const u32x4_t v, uint32_t* packed_out, int* scale_out)
{
    const uint32_t d[4] = {v[0], v[1], v[2], v[3]};
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = d[i] & 0x7FFFu, hi = (d[i] >> 16) & 0x7FFFu;
        amax = max(amax, max(lo, hi));
    }
    // block maximum over the 4 lanes of the quad (BF16 magnitude order = integer order)
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0xB1, 0xF, 0xF, false));
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4E, 0xF, 0xF, false));

    uint32_t packed = 0;
    int scale_byte;
    if (amax >= 0x7F80u) {
        scale_byte = 0xFF;                           // NaN or Inf in the block
    } else {
        scale_byte = (int)(amax >> 7) - 2;           // biased exponent of amax, minus 2
        scale_byte = scale_byte < 0 ? 0 : scale_byte;
        if constexpr (kHw) {
            // the convert divides by 2^(exponent field - 127) of its scale operand (field 0 is 2^-127)
            const float scale = __uint_as_float((uint32_t)scale_byte << 23);
            const uint32_t d0 = d[0], d1 = d[1], d2 = d[2], d3 = d[3];
            packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, __builtin_bit_cast(bf16x2_t, d0), scale, 0);
            packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, __builtin_bit_cast(bf16x2_t, d1), scale, 1);
            packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, __builtin_bit_cast(bf16x2_t, d2), scale, 2);
            packed = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(packed, __builtin_bit_cast(bf16x2_t, d3), scale, 3);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t lo = d[i] & 0xFFFFu, hi = d[i] >> 16;
                const uint32_t nlo = quantise_e2m1(lo & 0x7FFFu, scale_byte) | ((lo >> 15) << 3);
                const uint32_t nhi = quantise_e2m1(hi & 0x7FFFu, scale_byte) | ((hi >> 15) << 3);
                packed |= (nlo | (nhi << 4)) << (8 * i);
            }
        }
    }
    *packed_out = packed;
    *scale_out = scale_byte;
}

}  // namespace mxfp4
