// What the two kernels of the 8-bit product share (gemm_a8.hip: few rows, gemm_a8_block.hip: many).
#pragma once

#include "common.h"
#include "layer.h"
#include "../../include/mxfp4.h"

namespace mxfp4 {
namespace a8 {

typedef __attribute__((ext_vector_type(8))) int i32x8_t;

constexpr int kOob = 0x7FFFFFF0;        // lane offset beyond any descriptor: the load returns zero

// 0 where at <= last, else an offset beyond any descriptor (arithmetic, as a branch around a load makes the compiler wait for it).
__device__ __forceinline__ int past(int last, int at) { return ((last - at) >> 31) & kOob; }

__device__ __forceinline__ f32x4_t mfma(u32x4_t w, const u32x4_t* x, f32x4_t sum, uint32_t ws, uint32_t xs)
{
    const i32x8_t a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    const i32x8_t b = {(int)x[0][0], (int)x[0][1], (int)x[0][2], (int)x[0][3], (int)x[1][0], (int)x[1][1], (int)x[1][2], (int)x[1][3]};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, sum, 4, 0, 0, (int)ws, 0, (int)xs);
}

// Four finished sums of row m, weight rows n .. n + 3 (n a multiple of 4), on their way out.
struct Out {
    const uint16_t* bias;
    const uint16_t* residual;
    uint16_t* y;
    int64_t ldy, ldr;
    int m, n, act;
};

__device__ __forceinline__ void finish(const Out& o, int m, int n, f32x4_t z)
{
    if (m >= o.m || n >= o.n)
        return;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (o.bias && n + i < o.n)
            z[i] += bf16_bits_to_f32(o.bias[n + i]);
    if (o.act == MXFP4_ACT_SWIGLU) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            if (n + i >= o.n)
                break;
            const int c = (n + i) >> 1;
            float t = silu_gate(z[i], z[i + 1]);
            if (o.residual)
                t += bf16_bits_to_f32(o.residual[m * o.ldr + c]);
            o.y[m * o.ldy + c] = f32_to_bf16_rne(t);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (n + i >= o.n)
            break;
        if (o.residual)
            z[i] += bf16_bits_to_f32(o.residual[m * o.ldr + n + i]);
        o.y[m * o.ldy + n + i] = f32_to_bf16_rne(z[i]);
    }
}

// The blocks of many rows, by shape: 256 x 256, 128 x 256, 128 x 128, 64 x 128 outputs.
hipError_t launch_block(const A8Args& a, int shape, hipStream_t stream);

}  // namespace a8
}  // namespace mxfp4
