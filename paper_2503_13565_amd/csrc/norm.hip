// Root-mean-square norm of the residual stream with the addition in front of it:  h = x + r,  y = h / sqrt(mean(h^2) + eps) * w.
// h leaves as BF16 (the stream as the next layer reads it), y as BF16, as 8-bit blocks for the product of gemm_a8.hip, or as both.
//
// h stays in FP32 between the addition and y, so that y is rounded once; the 8-bit codes are those of the cast of the BF16 y, so that a
// caller who casts BF16 rows gets the same bits.  A row is read once: its T threads hold it in registers (C chunks of 8 elements each),
// the sum of squares goes through the vector unit's lane moves and, where a row has several waves, once through the LDS.
//
// Bound by memory: 6001 x 8192 with a residual reads and writes 345 MB, 70 us at the rate of a copy that writes half of what it moves; here 62.6
// (two thirds are reads).
//
// Squares leave FP32's range before the values do (above 2^64 or with h = x + r beyond the largest number).  Where the sum says so the row
// is scaled by the power of two of its largest h, which y does not depend on: the rare row reads its inputs again, every other pays one comparison.
#include "cast_block8.h"
#include "common.h"
#include "layer.h"

namespace mxfp4 {

namespace {

constexpr float kSmall = 0x1p-90f;      // sums of squares below this may have lost squares that matter...
constexpr float kSmallEps = 0x1p-60f;   // ...beside an eps below this

// Sum (or maximum) over the T threads of a row, in a fixed order; all of them return it.
template <int T, bool kMax>
__device__ __forceinline__ float row_reduce(float v, float* lds)
{
    auto join = [](float a, float b) { return kMax ? fmaxf(a, b) : a + b; };
    v = join(v, dpp_f32<0xB1>(v));
    v = join(v, dpp_f32<0x4E>(v));
    v = join(v, dpp_f32<0x141>(v));
    v = join(v, dpp_f32<0x140>(v));
    if constexpr (T >= 64) {
        auto pair = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
        v = join(__int_as_float(pair[0]), __int_as_float(pair[1]));
        pair = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
        v = join(__int_as_float(pair[0]), __int_as_float(pair[1]));
    }
    if constexpr (T > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
            lds[wave] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int i = 1; i < T / 64; ++i)
            v = join(v, lds[i]);
        __syncthreads();                // (the LDS is used again)
    }
    return v;
}

__device__ __forceinline__ float low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float high(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

template <int T, int C>
__global__ __launch_bounds__(T <= 64 ? 256 : T) void rms_norm_kernel(NormArgs a, float inverse_k)
{
    constexpr int R = T <= 64 ? 256 / T : 1;                    // rows of a workgroup
    __shared__ float lds[T > 64 ? T / 64 : 1];
    const int t = threadIdx.x % T, chunks = a.k >> 3;
    const int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / T;
    if (row >= a.m)
        return;                                                 // (whole rows: nothing below crosses a row unless it has the workgroup)
    const uint16_t* x = a.x + row * a.ldx;
    const uint16_t* r = a.r ? a.r + row * a.ldr : nullptr;
    auto chunk = [](const uint16_t* p, int c) { return *reinterpret_cast<const u32x4_t*>(p + (int64_t)c * 8); };

    // All loads at once: without conditions (a branch each, with a wait at its end), what is not there read from x and replaced.
    const uint16_t *r_at = r ? r : x, *w_at = a.w ? a.w : x;
    float h[C][8];
    u32x4_t w[C], vs[C], us[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int c = min(t + i * T, chunks - 1);
        vs[i] = chunk(x, c);
        us[i] = chunk(r_at, c);
        w[i] = chunk(w_at, c);
    }
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const bool inside = t + i * T < chunks;
        const u32x4_t none = {0, 0, 0, 0}, ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
        const u32x4_t v = inside ? vs[i] : none, u = inside && r ? us[i] : none;
        w[i] = a.w ? w[i] : ones;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[i][2 * e] = low(v[e]);
            h[i][2 * e + 1] = high(v[e]);
            if (r) {                                            // (not without one: -0 + 0 is 0)
                h[i][2 * e] += low(u[e]);
                h[i][2 * e + 1] += high(u[e]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            ss = fmaf(h[i][e], h[i][e], ss);
    ss = row_reduce<T, false>(ss, lds);

    float factor = 1.f, inv;
    u32x4_t sums[C];                                            // (h, before a rare row is scaled)
    if (a.sum)
#pragma unroll
        for (int i = 0; i < C; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sums[i][e] = f32_to_bf16_rne2(h[i][2 * e], h[i][2 * e + 1]);
    const float mean = fmaf(ss, inverse_k, a.eps);              // (infinite or NaN where ss is, and where only the addition of eps leaves FP32)
    inv = rsqrtf(mean);
    if (!(mean < INFINITY) || (ss < kSmall && a.eps < kSmallEps)) {
        // From h / 2, which no addition brings out of FP32 and which is exact where h is: the power of two has to follow h, not x and r, as these may cancel.
        const auto half = [](float v, float u) { return fmaf(u, 0.5f, v * 0.5f); };
        float top = 0.f;
        for (int c = t; c < chunks; c += T) {
            const u32x4_t v = chunk(x, c), u = r ? chunk(r, c) : u32x4_t{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
            for (int e = 0; e < 4; ++e)
                top = fmaxf(top, fmaxf(fabsf(half(low(v[e]), low(u[e]))), fabsf(half(high(v[e]), high(u[e])))));
        }
        top = row_reduce<T, true>(top, lds);
        // 2^-126 .. 2^126; a row with infinities has them in its sums, a row of NaN keeps them (the maximum leaves NaN out)
        const int exponent = (int)(__float_as_uint(top) >> 23);
        factor = __uint_as_float((uint32_t)min(max(254 - exponent, 1), 253) << 23);
        const float eps = a.eps * (0.5f * factor) * (0.5f * factor);
        if (top > 0.f && eps < INFINITY) {
            float s2 = 0.f;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const int c = t + i * T;
                u32x4_t v = {0, 0, 0, 0}, u = {0, 0, 0, 0};
                if (c < chunks) {
                    v = chunk(x, c);
                    u = r ? chunk(r, c) : u32x4_t{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};      // (-0, which changes nothing)
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    h[i][2 * e] = half(low(v[e]), low(u[e])) * factor;
                    h[i][2 * e + 1] = half(high(v[e]), high(u[e])) * factor;
                    s2 = fmaf(h[i][2 * e], h[i][2 * e], s2);
                    s2 = fmaf(h[i][2 * e + 1], h[i][2 * e + 1], s2);
                }
            }
            s2 = row_reduce<T, false>(s2, lds);
            inv = rsqrtf(fmaf(s2, inverse_k, eps));
        }
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int c = t + i * T;
        u32x4_t y;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = f32_to_bf16_rne2(h[i][2 * e] * inv * low(w[i][e]), h[i][2 * e + 1] * inv * high(w[i][e]));
        if (c < chunks) {                                       // (quads of lanes are inside or outside together where K % 32 = 0)
            if (a.sum)
                *reinterpret_cast<u32x4_t*>(a.sum + row * a.lds + (int64_t)c * 8) = sums[i];
            if (a.y)
                *reinterpret_cast<u32x4_t*>(a.y + row * a.ldy + (int64_t)c * 8) = y;
            if (a.q8) {
                u32x2_t code;
                int scale;
                cast_group8<true>(y, &code, &scale);
                *reinterpret_cast<u32x2_t*>(a.q8 + row * a.k + (int64_t)c * 8) = code;
                if ((c & 3) == 0)
                    a.s[row * (a.k >> 5) + (c >> 2)] = (uint8_t)scale;
            }
        }
    }
}

// The launch's grid holds less than 2^32 threads, so very many rows are several launches.
template <int T, int C>
hipError_t launch(NormArgs a, hipStream_t stream)
{
    constexpr int R = T <= 64 ? 256 / T : 1, kMost = 1 << 21;
    for (int64_t left = a.m;;) {
        a.m = (int)(left < kMost ? left : kMost);
        rms_norm_kernel<T, C><<<dim3((unsigned)((a.m + R - 1) / R)), T <= 64 ? 256 : T, 0, stream>>>(a, 1.f / (float)a.k);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || (left -= a.m) == 0)
            return e;
        a.x += kMost * a.ldx;
        a.r = a.r ? a.r + kMost * a.ldr : nullptr;
        a.sum = a.sum ? a.sum + kMost * a.lds : nullptr;
        a.y = a.y ? a.y + kMost * a.ldy : nullptr;
        a.q8 = a.q8 ? a.q8 + (int64_t)kMost * a.k : nullptr;
        a.s = a.s ? a.s + (int64_t)kMost * (a.k >> 5) : nullptr;
    }
}

}  // namespace

hipError_t launch_rms_norm(const NormArgs& a, hipStream_t stream)
{
    const int chunks = a.k >> 3;
    if (chunks <= 16)
        return launch<16, 1>(a, stream);
    if (chunks <= 64)
        return launch<64, 1>(a, stream);
    // A thread per chunk where rows are few (one row of 4096: 1.8 us, and 2.1 with two chunks a thread), two chunks a thread where every unit
    // has rows (6001 x 8192 with a residual and 8-bit rows: 62.6 us, and 70.0 with one, 63.8 with four).
    const bool many = a.m >= 256;
    if (chunks <= 256)
        return many ? launch<128, 2>(a, stream) : launch<256, 1>(a, stream);
    if (chunks <= 512)
        return many ? launch<256, 2>(a, stream) : launch<512, 1>(a, stream);
    if (chunks <= 1024)
        return many ? launch<512, 2>(a, stream) : launch<1024, 1>(a, stream);
    if (chunks <= 2048)
        return launch<1024, 2>(a, stream);
    return launch<1024, 8>(a, stream);
}

}  // namespace mxfp4
