// What the kernels of the 8-bit product share (gemm_a8.hip: few rows, gemm_a8_mid.hip: some tens to hundreds, gemm_a8_block.hip: many).
#pragma once

#include <utility>

#include "a8_stage.h"
#include "common.h"
#include "layer.h"
#include "../../include/mxfp4.h"

namespace mxfp4 {
namespace a8 {

typedef __attribute__((ext_vector_type(8))) int i32x8_t;

__device__ __forceinline__ f32x4_t mfma(u32x4_t w, const u32x4_t* x, f32x4_t sum, uint32_t ws, uint32_t xs)
{
    const i32x8_t a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    const i32x8_t b = {(int)x[0][0], (int)x[0][1], (int)x[0][2], (int)x[0][3], (int)x[1][0], (int)x[1][1], (int)x[1][2], (int)x[1][3]};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, sum, 4, 0, 0, (int)ws, 0, (int)xs);
}

// A buffer descriptor in scalar registers, for assembly.
__device__ __forceinline__ u32x4_t words(const uint8_t* p, int bytes)
{
    auto uniform = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return u32x4_t{uniform((uint32_t)a), uniform((uint32_t)(a >> 32) & 0xFFFFu), uniform((uint32_t)bytes), 0x00020000u};
}

__device__ __forceinline__ uint32_t lds_address(const uint8_t* p)
{
    return (uint32_t)reinterpret_cast<uint64_t>((__attribute__((address_space(3))) const uint8_t*)p);
}

// 16 bytes a lane from memory into the LDS, lane after lane from `to` on; zeros where the offset is past the descriptor.  m0 holds where
// lane 0's bytes go.  The load reads scalar registers that a vector instruction may have written just in front: five wait states, which the
// compiler does not count into assembly.  Nor does it count the load: a wait for vector memory stands wherever the LDS is read.
__device__ __forceinline__ void direct(uint32_t to, int off, const u32x4_t& r, int from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(r), "s"(from)
                 : "memory", "m0");
}

// silu(g) * u as common.h has it, with the hardware's reciprocal (off by one step) in place of the division, whose ten instructions for every
// output are 18 of the 337 us that 4003 rows x 22016 x 4096 took with it.  The reciprocal gives no subnormal numbers, and 1 + e^-g may be more than 2^126: a
// quarter of it is not, so silu is there down to where e^-g leaves FP32 (g = -88.7; 0 from there on, as with the division).
__device__ __forceinline__ float gate_of(float g, float u)
{
    return g * (0.25f * __builtin_amdgcn_rcpf(fmaf(__expf(-g), 0.25f, 0.25f))) * u;
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
            float t = gate_of(z[i], z[i + 1]);
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

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

// Matrix instructions run with all lanes.  Where their result is used under a condition, the compiler may move them behind it, and the operands of
// the other lanes with it; this keeps them in front.
__device__ __forceinline__ void settle(f32x16_t& v) { asm volatile("" : "+v"(v)); }

template <class F, int... I>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F f)
{
    each_of(f, std::make_integer_sequence<int, N>{});
}

// Up to eight finished outputs of row m from column c on (a multiple of 8 of o's columns), before the residual.  wide: rows' pieces
// of 16 bytes are aligned.
__device__ __forceinline__ void finish8(const Out& o, bool wide, int m, int c, int columns, float* t)
{
    if (wide && c + 8 <= columns) {
        u32x4_t v;
        if (o.residual) {
            v = *reinterpret_cast<const u32x4_t*>(o.residual + m * o.ldr + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                t[2 * e] += __uint_as_float(v[e] << 16);
                t[2 * e + 1] += __uint_as_float(v[e] & 0xFFFF0000u);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = f32_to_bf16_rne2(t[2 * e], t[2 * e + 1]);
        *reinterpret_cast<u32x4_t*>(o.y + m * o.ldy + c) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + e < columns)
            o.y[m * o.ldy + c + e] = f32_to_bf16_rne(o.residual ? t[e] + bf16_bits_to_f32(o.residual[m * o.ldr + c + e]) : t[e]);
}

// A wave's MF x NF tiles of 32 x 32 sums on their way out through a part of the LDS of its own, 32 rows at a time, so that whole pieces of
// rows are stored.  Lane i + 32 h holds, of row i of a tile, the 16 sums from 16 h on.
constexpr int leave_stride(int nf) { return 32 * nf + 4; }
constexpr int leave_bytes(int nf) { return 8 * 32 * leave_stride(nf) * 4; }                  // of eight waves

// A piece of row m, weight rows from n on: the sums of eight outputs, or with the gate sixteen sums of eight, as WK parts `stride` floats apart.
template <int WK>
__device__ __forceinline__ void finish_piece(const Out& o, bool wide, int m, int n, const float* from, int stride)
{
    const bool gate = o.act == MXFP4_ACT_SWIGLU;
    float z[16];
#pragma unroll
    for (int e = 0; e < 16; e += 4) {
        if (e < 8 || gate) {
            f32x4_t v = *reinterpret_cast<const f32x4_t*>(from + e);
#pragma unroll
            for (int w = 1; w < WK; ++w)
                v += *reinterpret_cast<const f32x4_t*>(from + w * stride + e);
            z[e] = v[0], z[e + 1] = v[1], z[e + 2] = v[2], z[e + 3] = v[3];
        }
    }
    if (o.bias)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if ((e < 8 || gate) && n + e < o.n)
                z[e] += bf16_bits_to_f32(o.bias[n + e]);
    if (gate)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            z[e] = gate_of(z[2 * e], z[2 * e + 1]);
    finish8(o, wide, m, gate ? n >> 1 : n, gate ? o.n >> 1 : o.n, z);
}

template <int MF, int NF>
__device__ __forceinline__ void leave(const Out& o, bool wide, uint8_t* lds, int lane, int m0, int n0, const f32x16_t (&acc)[MF][NF])
{
    constexpr int kStride = leave_stride(NF);
    float* tile = reinterpret_cast<float*>(lds);
    const int piece = o.act == MXFP4_ACT_SWIGLU ? 16 : 8, pieces = 32 * NF / piece;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4_t*>(tile + (lane & 31) * kStride + f * 32 + 16 * (lane >> 5) + e) =
                    f32x4_t{acc[i][f][e], acc[i][f][e + 1], acc[i][f][e + 2], acc[i][f][e + 3]};
        const int m1 = m0 + i * 32;
#pragma unroll 1
        for (int at = lane; at < 32 * pieces; at += 64) {
            const int row = at / pieces, n = at % pieces * piece;
            if (m1 + row < o.m && n0 + n < o.n)
                finish_piece<1>(o, wide, m1 + row, n0 + n, tile + row * kStride + n, 0);
        }
    }
}

// Whether rows' pieces of 16 bytes are aligned, of y and the residual.
inline bool wide_rows(const A8Args& a)
{
    auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    return aligned(a.y) && a.ldy % 8 == 0 && aligned(a.epi.residual) && (!a.epi.residual || a.ldr % 8 == 0);
}

// The way out of the rows from `at` on, `m` of them.
inline Out out_of(const A8Args& a, int64_t at, int m)
{
    return {a.epi.bias, a.epi.residual ? a.epi.residual + at * a.ldr : nullptr, a.y + at * a.ldy, a.ldy, a.ldr, m, a.n, a.epi.act};
}

// The kernels' shapes, by the outputs of a workgroup.
enum Shape { kRows1, kRows4, kRows8, kRows12, kRows16, kRows16Deep, kRows32, kMid32x64, kMid32x64Deep, kMid64x128, kMid128x128, kBlock128x256, kBlock256x256 };
hipError_t launch_mid(const A8Args& a, Shape shape, hipStream_t stream);
hipError_t launch_block(const A8Args& a, Shape shape, hipStream_t stream);

}  // namespace a8
}  // namespace mxfp4
