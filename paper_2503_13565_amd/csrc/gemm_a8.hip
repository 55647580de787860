// The product of 8-bit rows with MXFP4 weights, y = x8 * dequant(W)^T, on the scaled matrix instructions: E4M3 codes against E2M1 codes,
// each block of 32 with its scale byte, exactly as both lie in memory (arXiv 2503.13565, section 3.4.3, Eq. 2 with 8-bit rows in place
// of BF16).  Nothing is decoded, and an instruction does four times the work of a BF16 one in twice its time.
//
// v_mfma_scale_f32_16x16x128_f8f6f4, one step of 128 along K: lane i + 16 g holds, of row i,
//   weights (A)      16 bytes: block g of the step,
//   activations (B)  16 bytes from 16 g on and 16 bytes from 64 + 16 g on,
//   scales           the byte of block g, of either operand.
// The sums: row i of x, weight rows 4 g .. 4 g + 3.
#include "gemm_a8.h"

namespace mxfp4 {
namespace a8 {

namespace {

// A workgroup computes 16 MF rows of x times 16 NF weight rows; its eight waves share the steps of K, and both operands go straight to
// the registers.  The waves' sums meet in the LDS and are added in wave order.
template <int MF, int NF, bool kRagged>
__global__ __launch_bounds__(512) void w4a8_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xs,
                                                   const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, int k, int tiles_m, Out out)
{
    constexpr int BM = MF * 16, BN = NF * 16, D = 2;
    __shared__ f32x4_t red[8][MF * NF][64];
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m0 = (int)(blockIdx.x % tiles_m) * BM, n0 = (int)(blockIdx.x / tiles_m) * BN;
    const int rows = min(BM, out.m - m0), cols = min(BN, out.n - n0);
    const int nblk = k >> 5, steps = (k + 127) >> 7;
    auto view = [](const uint8_t* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p), 0, bytes, 0x00020000); };
    const __amdgpu_buffer_rsrc_t rx = view(x + (int64_t)m0 * k, rows * k), rxs = view(xs + (int64_t)m0 * nblk, rows * nblk);
    const __amdgpu_buffer_rsrc_t rq = view(q + (int64_t)n0 * (k >> 1), cols * (k >> 1)), rs = view(s + (int64_t)n0 * nblk, cols * nblk);

    struct Slot {
        u32x4_t w[NF], x[MF][2];
        uint32_t ws[NF], xs[MF];
    };
    Slot slot[D];
    // What lies past K, or past the last row, loads as zeros under the scale 2^-127.
    auto issue = [&](Slot& v, int T) {
        const int p_w = past(nblk - 1, 4 * T + lg), p_lo = past((k >> 4) - 1, 8 * T + lg), p_hi = past((k >> 4) - 1, 8 * T + 4 + lg);
        const int p_s = kRagged ? p_w : past(steps - 1, T);
        auto scale = [&](const __amdgpu_buffer_rsrc_t r, int off) {
            return kRagged ? (uint32_t)__builtin_amdgcn_raw_buffer_load_b8(r, (off + 4 * T + lg) | p_s, 0, 0)
                           : (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(r, (off + 4 * T) | p_s, 0, 0);
        };
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int row = f * 16 + li, gone = past(cols - 1, row);
            v.w[f] = __builtin_amdgcn_raw_buffer_load_b128(rq, (row * (k >> 1) + T * 64 + lg * 16) | p_w | gone, 0, 0);
            v.ws[f] = scale(rs, (row * nblk) | gone);
        }
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            const int row = f * 16 + li, gone = past(rows - 1, row);
            v.x[f][0] = __builtin_amdgcn_raw_buffer_load_b128(rx, (row * k + T * 128 + lg * 16) | p_lo | gone, 0, 0);
            v.x[f][1] = __builtin_amdgcn_raw_buffer_load_b128(rx, (row * k + T * 128 + 64 + lg * 16) | p_hi | gone, 0, 0);
            v.xs[f] = scale(rxs, (row * nblk) | gone);
        }
    };
    f32x4_t acc[MF][NF] = {};
    auto multiply = [&](const Slot& v) {
#pragma unroll
        for (int a = 0; a < MF; ++a)
#pragma unroll
            for (int b = 0; b < NF; ++b)
                acc[a][b] = mfma(v.w[b], v.x[a], acc[a][b], kRagged ? v.ws[b] : v.ws[b] >> (8 * lg), kRagged ? v.xs[a] : v.xs[a] >> (8 * lg));
    };
    int T = wave;
#pragma unroll
    for (int d = 0; d < D; ++d)
        issue(slot[d], T + 8 * d);
    for (; T < steps; T += 8 * D) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            multiply(slot[d]);
            issue(slot[d], T + 8 * (d + D));
        }
    }
#pragma unroll
    for (int a = 0; a < MF; ++a)
#pragma unroll
        for (int b = 0; b < NF; ++b)
            red[wave][a * NF + b][lane] = acc[a][b];
    __syncthreads();
    for (int i = threadIdx.x; i < MF * NF * 64; i += 512) {
        const int f = i >> 6, l = i & 63;
        f32x4_t z = red[0][f][l];
#pragma unroll
        for (int w = 1; w < 8; ++w)
            z += red[w][f][l];
        finish(out, m0 + f / NF * 16 + (l & 15), n0 + f % NF * 16 + 4 * (l >> 4), z);
    }
}

// A grid holds less than 2^32 threads, so very many rows are several launches.
template <int MF, int NF, bool kRagged>
hipError_t launch(const A8Args& a, hipStream_t stream)
{
    const int64_t tiles_n = (a.n + NF * 16 - 1) / (NF * 16), most = max(((int64_t)1 << 22) / tiles_n, (int64_t)1) * (MF * 16);
    for (int64_t at = 0; at < a.m; at += most) {
        const int m = (int)min(most, a.m - at), tiles_m = (m + MF * 16 - 1) / (MF * 16);
        const Out out = {a.epi.bias, a.epi.residual ? a.epi.residual + at * a.ldr : nullptr, a.y + at * a.ldy, a.ldy, a.ldr, m, a.n, a.epi.act};
        w4a8_kernel<MF, NF, kRagged><<<dim3((unsigned)(tiles_m * tiles_n)), 512, 0, stream>>>(
            a.x + at * a.k, a.xs + at * (a.k >> 5), a.q, a.s, a.k, tiles_m, out);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace

}  // namespace a8

hipError_t launch_w4a8(const A8Args& a, const DeviceInfo&, hipStream_t stream)
{
    const bool ragged = a.k % 128 != 0;
    if (const char* e = knob("MXFP4_A8_SHAPE")) {
        if (atoi(e) >= 0)
            return a8::launch_block(a, atoi(e), stream);
    } else if (a.m > 64) {
        return a8::launch_block(a, a.m > 512 ? 0 : a.m > 128 ? 1 : a.m > 64 ? 2 : 3, stream);
    }
    if (a.m <= 16)
        return ragged ? a8::launch<1, 1, true>(a, stream) : a8::launch<1, 1, false>(a, stream);
    if (a.m <= 32)
        return ragged ? a8::launch<2, 1, true>(a, stream) : a8::launch<2, 1, false>(a, stream);
    return ragged ? a8::launch<4, 2, true>(a, stream) : a8::launch<4, 2, false>(a, stream);
}

}  // namespace mxfp4
