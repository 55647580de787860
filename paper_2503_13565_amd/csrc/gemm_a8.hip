// The product of 8-bit rows with MXFP4 weights, y = x8 * dequant(W)^T, on the scaled matrix instructions: E4M3 codes against E2M1 codes,
// each block of 32 with its scale byte, exactly as both lie in memory (arXiv 2503.13565, section 3.4.3, Eq. 2 with 8-bit rows in place
// of BF16).  Nothing is decoded, and an instruction does four times the work of a BF16 one in twice its time.  This file has the kernel of
// few rows, where the weights' way from memory is what there is to do; gemm_a8_block.hip has many.
//
// v_mfma_scale_f32_16x16x128_f8f6f4, one step of 128 along K: lane i + 16 g holds, of row i,
//   weights (A)      16 bytes: block g of the step,
//   activations (B)  16 bytes from 16 g on and 16 bytes from 64 + 16 g on,
//   scales           the byte of block g, of either operand.
// The sums: row i of x, weight rows 4 g .. 4 g + 3.  (How the instruction adds: include/mxfp4.h, mxfp4_w4a8_gemm.)
//
// A workgroup has 16 NF weight rows and all rows of x (up to 16 WM MF of them), and its eight waves are WM x WK: WK share the steps of K.  K goes
// by in phases of WK steps.  Both operands of a phase lie in the LDS as rows, brought there by loads that write it directly, whole lines of memory an
// instruction (loads in the layout of the matrix instruction touch a line per lane: 77 rows x 4096 x 11008 33 us), D - 1 phases ahead.  The
// partial sums of the WK waves meet in the LDS at the end and are added in wave order.
//   - Chunk c (16 bytes) of row r lies at c ^ (r % 16): the sixteen lanes that a turn of the LDS serves find sixteen different places.
//   - XR rows of x are held; with fewer than 16, the instruction's other columns read them again, and are not stored.
//   - The scale bytes of the workgroup's rows are one piece of memory, which is copied at the start; a lane reads its byte.
//   - What lies past K loads as zeros, under the row's last scale (which is NaN only where the row is).
// Bound by the start, the first loads and the last sums of a workgroup, and by the weights' way from memory: one row x 12288 x 4096 7.2 us, 8.4 where the weights
// are in no cache (27 MB, 3.8 us at the rate of a kernel that only reads; the decode kernel of BF16 rows 6.7), nine rows x 22016 x 4096 with the gate 10.5 and
// 12.4 (48 MB, 6.9).
#include "gemm_a8.h"

namespace mxfp4 {
namespace a8 {

namespace {

constexpr int rows_buffer(int wk, int xr, int bn) { return wk * (xr * 128 + bn * 64); }
constexpr int rows_scales(int rows, int nblk) { return (rows * nblk + 1023) / 1024 * 1024; }
// D buffers (afterwards: the waves' sums), a KiB that surplus loads write, the scales
constexpr int rows_fixed(int wk, int mf, int nf, int xr, int bn, int d)
{
    const int buffers = d * rows_buffer(wk, xr, bn), sums = 8 * mf * nf * 1024;
    return (buffers > sums ? buffers : sums) + 1024;
}
template <int WM, int WN, int WK, int MF, int NF, int XR, int D>
__global__ __launch_bounds__(512) void w4a8_rows_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xs,
                                                        const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, int k, int tiles_m, Out out)
{
    static_assert(WM * WN * WK == 8 && (XR == WM * MF * 16 || (WM * MF == 1 && XR < 16)), "eight waves; the rows of x");
    constexpr int BM = WM * MF * 16, BN = WN * NF * 16;
    constexpr int kX = XR * WK / 8, kW = BN * WK / 16, kUnits = kX + kW, C = (kUnits + 7) / 8;     // KiB of a phase, loads of a wave
    static_assert(kX * 8 == XR * WK && kW * 16 == BN * WK, "whole KiB");
    constexpr int kBuf = rows_buffer(WK, XR, BN), kFixed = rows_fixed(WK, MF, NF, XR, BN, D);
    extern __shared__ __align__(16) uint8_t smem[];
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (WN * WK), wn = wave / WK % WN, wk = wave % WK;
    const int m0 = (int)(blockIdx.x % tiles_m) * BM, n0 = (int)(blockIdx.x / tiles_m) * BN;
    const int rows = min(BM, out.m - m0), cols = min(BN, out.n - n0);
    const int nblk = k >> 5, steps = (k + 127) >> 7, phases = (steps + WK - 1) / WK;
    const u32x4_t rx = words(x + (int64_t)m0 * k, rows * k), rq = words(q + (int64_t)n0 * (k >> 1), cols * (k >> 1));
    const uint32_t lds_at = lds_address(smem);

    // Load c of wave w fills KiB 8 c + w of a phase: x first, the weights behind it.
    int off[C], chunk[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int u = c * 8 + wave;
        const bool of_x = u < kX;
        const int piece = (of_x ? u : u - kX) * 64 + lane;
        chunk[c] = of_x ? piece_chunk(piece, WK * 8) : piece_chunk(piece, WK * 4);
        off[c] = u >= kUnits ? kOob : of_x ? piece_offset(piece, WK * 8, rows, k) : piece_offset(piece, WK * 4, cols, k >> 1);
    }
    auto issue = [&](int p, int b) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int u = c * 8 + wave, t = p * WK;
            if (u < kX)
                direct(lds_at + b * kBuf + u * 1024, off[c] | past((k >> 4) - 1, phase_chunk(t, 128) + chunk[c]), rx, phase_from(t, steps, 128));
            else
                direct(lds_at + (u < kUnits ? b * kBuf + u * 1024 : kFixed - 1024), off[c] | past(nblk - 1, phase_chunk(t, 64) + chunk[c]), rq,
                       phase_from(t, steps, 64));
        }
    };

    // Where a row has whole chunks of scales, row r's are turned by r of them: rows of 128 bytes would have their bytes of a step in one bank (nine
    // rows x 22016 x 4096 with the gate 10.6 us, 10.9 unturned).  Divisions by their number as products with `inverse` (numbers far below 2^16).
    const bool turns = (nblk & 15) == 0 && nblk > 16;
    const int around = turns ? nblk >> 4 : 1 << 20;
    const uint32_t inverse = turns ? (uint32_t)(0x100000000ull / (uint32_t)around) + 1 : 0;
    const auto turned = [&](int row) { return turns ? row - (int)__umulhi((uint32_t)row, inverse) * around : 0; };
    const int ws_bytes = rows_scales(BN, nblk), xs_bytes = rows_scales(XR, nblk);
    {
        // (a load is in range by whole dwords: the last one, which holds the last byte, counts)
        const u32x4_t rs = words(s + (int64_t)n0 * nblk, (cols * nblk + 3) & ~3), rxs = words(xs + (int64_t)m0 * nblk, (rows * nblk + 3) & ~3);
        const auto from = [&](int u) {
            const int at = u * 64 + lane, row = (int)__umulhi((uint32_t)at, inverse), c = at - row * around;
            return turns ? (at - c + (c - turned(row) + (c < turned(row) ? around : 0))) * 16 : at * 16;
        };
        for (int u = wave; u * 1024 < ws_bytes; u += 8)
            direct(lds_at + kFixed + u * 1024, from(u), rs, 0);
        for (int u = wave; u * 1024 < xs_bytes; u += 8)
            direct(lds_at + kFixed + ws_bytes + u * 1024, from(u), rxs, 0);
    }
#pragma unroll
    for (int d = 0; d < D - 1; ++d)
        issue(d, d);

    const int xrow = XR < 16 ? min(li, XR - 1) : wm * MF * 16 + li, wrow = wn * NF * 16 + li;
    const int x_lo = xrow * (WK * 128) + ((8 * wk + lg) ^ turn(xrow, WK * 8)) * 16;
    const int x_hi = xrow * (WK * 128) + ((8 * wk + 4 + lg) ^ turn(xrow, WK * 8)) * 16;
    const int w_at = kX * 1024 + wrow * (WK * 64) + ((4 * wk + lg) ^ turn(wrow, WK * 4)) * 16;
    const uint8_t *sw = smem + kFixed + wrow * nblk, *sx = smem + kFixed + ws_bytes + xrow * nblk;
    const auto byte = [&](int row, int block) {
        const int c = (block >> 4) + turned(row);
        return (c >= around ? c - around : c) * 16 + (block & 15);
    };
    f32x4_t acc[MF][NF] = {};
    int b = 0;
    for (int p = 0; p < phases; ++p) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 2) * C) : "memory");      // (D - 2 phases are younger than this one)
        lds_barrier();
        issue(p + D - 1, b == 0 ? D - 1 : b - 1);               // into the buffer that the phase before this one read
        const uint8_t* buf = smem + b * kBuf;
        const int block = min(4 * (p * WK + wk) + lg, nblk - 1);
        u32x4_t w[NF], v[MF][2];
        uint32_t ws[NF], vs[MF];
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            w[f] = *reinterpret_cast<const u32x4_t*>(buf + w_at + f * (16 * WK * 64));
            ws[f] = sw[f * 16 * nblk + byte(wrow + f * 16, block)];
        }
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            v[f][0] = *reinterpret_cast<const u32x4_t*>(buf + x_lo + f * (16 * WK * 128));
            v[f][1] = *reinterpret_cast<const u32x4_t*>(buf + x_hi + f * (16 * WK * 128));
            vs[f] = sx[f * 16 * nblk + byte(xrow + f * 16, block)];
        }
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int f = 0; f < NF; ++f)
                acc[i][f] = mfma(w[f], v[i], acc[i][f], ws[f], vs[i]);
        b = b == D - 1 ? 0 : b + 1;
    }

    drain_vmem();                                               // (the loads behind the last phase write the LDS)
    __syncthreads();
    f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < NF; ++f)
            red[((wk * WM + wm) * MF + i) * (WN * NF * 64) + (wn * NF + f) * 64 + lane] = acc[i][f];
    __syncthreads();
    constexpr int kSums = WM * MF * WN * NF * 64;
    for (int i = threadIdx.x; i < kSums; i += 512) {
        const int f = i >> 6, l = i & 63;
        f32x4_t z = red[i];
#pragma unroll
        for (int w = 1; w < WK; ++w)
            z += red[w * kSums + i];
        if (XR == BM || (l & 15) < XR)
            finish(out, m0 + f / (WN * NF) * 16 + (l & 15), n0 + f % (WN * NF) * 16 + 4 * (l >> 4), z);
    }
}

// A grid holds less than 2^32 threads, so very many rows are several launches.
template <int WM, int WN, int WK, int MF, int NF, int XR, int D>
hipError_t launch(const A8Args& a, hipStream_t stream)
{
    constexpr int BM = WM * MF * 16, BN = WN * NF * 16;
    const int nblk = a.k >> 5, lds = rows_fixed(WK, MF, NF, XR, BN, D) + rows_scales(BN, nblk) + rows_scales(XR, nblk);
    if (lds > 160 * 1024)                                       // (a K so long that the rows' scales leave no room)
        return launch_mid(a, kMid32x64, stream);
    static LdsLimit limit;
    const hipError_t raised = limit.raise(reinterpret_cast<const void*>(w4a8_rows_kernel<WM, WN, WK, MF, NF, XR, D>), 160 * 1024);
    if (raised != hipSuccess)
        return raised;
    const int64_t tiles_n = (a.n + BN - 1) / BN, most = max(((int64_t)1 << 22) / tiles_n, (int64_t)1) * BM;
    for (int64_t at = 0; at < a.m; at += most) {
        const int m = (int)min(most, a.m - at), tiles_m = (m + BM - 1) / BM;
        w4a8_rows_kernel<WM, WN, WK, MF, NF, XR, D><<<dim3((unsigned)(tiles_m * tiles_n)), 512, lds, stream>>>(
            a.x + at * a.k, a.xs + at * (a.k >> 5), a.q, a.s, a.k, tiles_m, out_of(a, at, m));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace

}  // namespace a8

namespace {

// Which shape a call takes.  Up to 16 rows: the kernel with that many rows in the LDS; from nine rows on one of 16 weight rows where their blocks fit
// the device twice (16 rows x 4096 x 4096 5.0 us, 6.8 in blocks of 32; 4096 x 11008 7.2 and 13.4), one of 32 beyond (12288 x 4096 8.3 us, 10.2;
// 22016 x 4096 at nine rows with the gate 11.6, 16.1).  More rows: the shape whose rounds take the least.  A round (as many blocks as the device holds)
// takes base + step for every 128 of K, in us, as measured on some seventy sizes from 17 x 23 x 128 to 4003 x 22016 x 4096: `few` with some tens of
// blocks, `full` with one on every unit, and the last two where two fit a unit and share it.
struct Rounds {
    a8::Shape shape;
    int bm, bn;
    float base, few, full;
    float base2, step2;
};
constexpr Rounds kRounds[] = {
    {a8::kRows32, 32, 32, 1.5f, 0.085f, 0.17f, 1.0f, 0.31f},
    {a8::kMid32x64, 32, 64, 2.9f, 0.115f, 0.17f, 1.5f, 0.28f},
    {a8::kMid32x64Deep, 32, 64, 2.9f, 0.115f, 0.15f, 0.f, 0.f},
    {a8::kMid64x128, 64, 128, 3.8f, 0.285f, 0.33f, 0.f, 0.f},
    {a8::kMid128x128, 128, 128, 5.7f, 0.43f, 0.55f, 0.f, 0.f},
    {a8::kBlock128x256, 128, 256, 7.5f, 0.745f, 0.80f, 7.0f, 1.45f},
    {a8::kBlock256x256, 256, 256, 12.5f, 1.06f, 1.20f, 0.f, 0.f},
};

float time_of(const Rounds& r, int64_t blocks, float steps, int cus)
{
    auto one = [&](int64_t some) { return some ? r.base + (r.few + (r.full - r.few) * (some < cus ? (float)some / cus : 1.f)) * steps : 0.f; };
    if (r.step2 == 0.f)
        return (float)(blocks / cus) * one(cus) + one(blocks % cus);
    const int64_t rest = blocks % (2 * cus);
    const float two = r.base2 + r.step2 * steps;
    return (float)(blocks / (2 * cus)) * two + (rest > cus ? two : one(rest));
}

a8::Shape shape_of(int64_t m, int64_t n, int64_t k, const DeviceInfo& dev)
{
    if (const char* e = knob("MXFP4_A8_SHAPE"))
        if (atoi(e) >= 0)
            return (a8::Shape)atoi(e);
    if (m <= 4)
        return m == 1 ? a8::kRows1 : a8::kRows4;
    if (m <= 8)
        return a8::kRows8;
    if (m <= 16)
        return n > (int64_t)32 * dev.cus ? a8::kRows16 : m <= 12 ? a8::kRows12 : a8::kRows16Deep;
    const float steps = (float)((k + 127) / 128);
    a8::Shape best = a8::kBlock256x256;
    float least = INFINITY;
    for (const Rounds& r : kRounds) {
        const float time = time_of(r, ((m + r.bm - 1) / r.bm) * ((n + r.bn - 1) / r.bn), steps, dev.cus);
        if (time < least) {
            least = time;
            best = r.shape;
        }
    }
    return best;
}

}  // namespace

hipError_t launch_w4a8(const A8Args& whole, const DeviceInfo& dev, hipStream_t stream)
{
    using namespace a8;
    // A grid holds less than 2^32 threads (a larger one is cut without an error), so very many weight rows are several launches: 2^26 of them are 2^22
    // workgroups of the narrowest blocks.  (Very many rows of x: each kernel's launch.)
    constexpr int kMost = 1 << 26;
    A8Args a = whole;
    for (int64_t at = 0; whole.n - at > kMost; at += kMost) {
        a.n = kMost;
        const hipError_t e = launch_w4a8(a, dev, stream);
        if (e != hipSuccess)
            return e;
        const int64_t columns = a.epi.act == MXFP4_ACT_SWIGLU ? kMost / 2 : kMost;
        a.q += (int64_t)kMost * (a.k >> 1);
        a.s += (int64_t)kMost * (a.k >> 5);
        a.epi.bias = a.epi.bias ? a.epi.bias + kMost : nullptr;
        a.epi.residual = a.epi.residual ? a.epi.residual + columns : nullptr;
        a.y += columns;
        a.n = (int)(whole.n - at - kMost);
    }
    const Shape shape = shape_of(a.m, a.n, a.k, dev);
    switch (shape) {
    case kRows1:
        return launch<1, 1, 8, 1, 1, 1, 3>(a, stream);
    case kRows4:
        return launch<1, 1, 8, 1, 1, 4, 3>(a, stream);
    case kRows8:
        return launch<1, 1, 8, 1, 1, 8, 3>(a, stream);
    case kRows12:
        return launch<1, 1, 8, 1, 1, 12, 3>(a, stream);
    case kRows16:
        return launch<1, 2, 4, 1, 1, 16, 2>(a, stream);
    case kRows16Deep:
        return launch<1, 1, 8, 1, 1, 16, 3>(a, stream);
    case kRows32:
        return launch<1, 2, 4, 2, 1, 32, 2>(a, stream);
    case kMid32x64:
    case kMid32x64Deep:
    case kMid64x128:
    case kMid128x128:
        return launch_mid(a, shape, stream);
    default:
        return launch_block(a, shape, stream);
    }
}

}  // namespace mxfp4
