// The product of 8-bit rows with MXFP4 weights for some tens to some hundreds of rows (gemm_a8.hip: fewer, gemm_a8_block.hip: more).
//
// The kernel of gemm_a8_block.hip in smaller blocks, of which one alone does not fill its compute unit's time: what bounds it is how long a
// step's operands are on their way.  So the loads leave D - 1 phases (of S steps each) ahead, and a phase waits for its own loads only, which
// takes scales that no wait of the compiler's stands in front of: they come into the LDS by direct loads too, sixteen steps at a time
// (64 bytes a row and up to 16 around them: a row of K / 32 bytes may start anywhere, a load starts at a dword), and a lane reads its byte
// (80 bytes from row to row, two lanes a bank).
//
// Where there are fewer blocks than compute units, K is cut into parts (grid y): the parts' sums go to the workspace in FP32, and a second kernel
// adds them in order.
#include "gemm_a8.h"

namespace mxfp4 {
namespace a8 {

namespace {

constexpr int mid_buffer(int bm, int bn, int s) { return s * (bm * 128 + bn * 64); }
constexpr int kScaleSteps = 16, kScaleRow = 80;
constexpr int scale_units(int rows) { return (rows * kScaleRow + 1023) / 1024; }
constexpr int phase_units(int bm, int bn, int s) { return (bm * s / 8 + bn * s / 16); }
// D phases, two times the scales of both operands' rows, and a KiB for the loads that a phase is short of
constexpr int mid_lds(int bm, int bn, int s, int d)
{
    return d * mid_buffer(bm, bn, s) + 2 * 1024 * (scale_units(bm) + scale_units(bn)) + (phase_units(bm, bn, s) % 8 ? 1024 : 0);
}

// part: null, or where this call's sums of its part of K go, [part][m][tiles_n * BN].
template <int WM, int WN, int MF, int NF, int S, int D>
__global__ __launch_bounds__(512, 2) void w4a8_mid_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xs,
                                                          const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, int k, int tiles_m,
                                                          int tiles_n, int part_steps, float* __restrict__ part, bool wide, Out out)
{
    static_assert(WM * WN == 8, "eight waves");
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32;
    constexpr int kBuf = mid_buffer(BM, BN, S), kX = BM * S / 8, kUnits = phase_units(BM, BN, S), C = (kUnits + 7) / 8;
    constexpr int kSx = scale_units(BM), kScaleUnits = kSx + scale_units(BN), kPhases = kScaleSteps / S;
    static_assert(mid_lds(BM, BN, S, D) <= 160 * 1024 && D <= kPhases, "the LDS; scales arrive before their steps");
    extern __shared__ __align__(16) uint8_t smem[];
    const int lane = threadIdx.x & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int nblk = k >> 5, t0 = blockIdx.y * part_steps, t1 = min(t0 + part_steps, (k + 127) >> 7);
    const int phases = (t1 - t0 + S - 1) / S, last_x = min(k >> 4, t1 * 8) - 1, last_w = min(nblk, t1 * 4) - 1;
    const int m0 = (int)(blockIdx.x % tiles_m) * BM, n0 = (int)(blockIdx.x / tiles_m) * BN;
    const int rows = min(BM, out.m - m0), cols = min(BN, out.n - n0);
    const u32x4_t rx = words(x + (int64_t)m0 * k, rows * k), rq = words(q + (int64_t)n0 * (k >> 1), cols * (k >> 1));
    // (a load is in range by whole dwords: the last one, which holds the last byte, counts)
    const u32x4_t rxs = words(xs + (int64_t)m0 * nblk, (rows * nblk + 3) & ~3), rs = words(s + (int64_t)n0 * nblk, (cols * nblk + 3) & ~3);
    const uint32_t lds_at = lds_address(smem);

    // Load c of wave w fills KiB 8 c + w of a phase: x first, the weights behind it.
    int off[C], chunk[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int u = c * 8 + wave;
        const bool of_x = u < kX;
        const int at = (of_x ? u : u - kX) * 64 + lane;
        const int row = of_x ? at / (S * 8) : at / (S * 4);
        chunk[c] = of_x ? at % (S * 8) ^ turn(row, S * 8) : at % (S * 4) ^ turn(row, S * 4);
        off[c] = u >= kUnits ? kOob : of_x ? (row * k + chunk[c] * 16) | past(rows - 1, row) : (row * (k >> 1) + chunk[c] * 16) | past(cols - 1, row);
    }
    auto issue = [&](int p, int b) {                            // (past the part's end: zeros, so that the loads of a phase are as many)
        const int t = p < phases ? t0 + p * S : t1;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int u = c * 8 + wave;
            if (u < kX)
                direct(lds_at + b * kBuf + u * 1024, off[c] | past(last_x, t * 8 + chunk[c]), rx, t * 128);
            else
                direct(lds_at + (u < kUnits ? b * kBuf + u * 1024 : D * kBuf + 2048 * kScaleUnits), off[c] | past(last_w, t * 4 + chunk[c]), rq, t * 64);
        }
    };
    auto issue_scales = [&](int part16) {                       // of the sixteen steps from t0 + 16 part16 on
#pragma unroll
        for (int c = 0; c < (kScaleUnits + 7) / 8; ++c) {
            const int u = c * 8 + wave;
            if (u < kScaleUnits) {
                const bool of_x = u < kSx;
                const int piece = (of_x ? u : u - kSx) * 64 + lane, row = piece / (kScaleRow / 16), at = piece % (kScaleRow / 16) * 16;
                const uint32_t to = lds_at + D * kBuf + ((part16 & 1) * kScaleUnits + u) * 1024;
                const int o = (((row * nblk + 4 * t0 + part16 * (4 * kScaleSteps)) & ~3) + at) | past((of_x ? rows : cols) - 1, row);
                if (of_x)
                    direct(to, o, rxs, 0);
                else
                    direct(to, o, rs, 0);
            }
        }
    };

    struct Half {
        u32x4_t x[MF][2], w[NF];
        uint32_t xs[MF], ws[NF];
    } half[2];
    const int wrow = 16 * (li >> 2 & 1) + 4 * (li >> 3) + (li & 3);
    const int x_row = wm * MF * 32 + li, w_row = wn * NF * 32 + wrow;
    const int x_read = x_row * (S * 128) + (lh ^ turn(x_row, S * 8)) * 16, w_read = kX * 1024 + w_row * (S * 64) + (lh ^ turn(w_row, S * 4)) * 16;
    int xs_read[MF], ws_read[NF];
#pragma unroll
    for (int f = 0; f < MF; ++f)
        xs_read[f] = D * kBuf + (x_row + f * 32) * kScaleRow + (((x_row + f * 32) * nblk) & 3);
#pragma unroll
    for (int f = 0; f < NF; ++f)
        ws_read[f] = D * kBuf + kSx * 1024 + (w_row + f * 32) * kScaleRow + (((w_row + f * 32) * nblk) & 3);
    auto read = [&](int p, int b, auto hh, Half& h) {           // half hh of phase p, in buffer b
        const uint8_t* buf = smem + b * kBuf;
        const int block = min(4 * (t0 + p * S) + 2 * hh + lh, nblk - 1) - 4 * t0, part16 = p / kPhases;
        const uint8_t* sc = smem + (part16 & 1) * (kScaleUnits * 1024) + min(max(block - part16 * (4 * kScaleSteps), 0), 4 * kScaleSteps - 1);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            h.w[f] = *reinterpret_cast<const u32x4_t*>(buf + (w_read ^ (hh * 32)) + f * (32 * S * 64));
            h.ws[f] = sc[ws_read[f]];
        }
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            h.x[f][0] = *reinterpret_cast<const u32x4_t*>(buf + (x_read ^ (hh * 64)) + f * (32 * S * 128));
            h.x[f][1] = *reinterpret_cast<const u32x4_t*>(buf + (x_read ^ (hh * 64 + 32)) + f * (32 * S * 128));
            h.xs[f] = sc[xs_read[f]];
        }
    };
    f32x16_t acc[MF][NF] = {};
    auto multiply = [&](const Half& h) {
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                const u32x4_t w = h.w[f], x0 = h.x[i][0], x1 = h.x[i][1];
                const i32x8_t A = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
                const i32x8_t B = {(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
                acc[i][f] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, acc[i][f], 4, 0, 0, (int)h.ws[f], 0, (int)h.xs[i]);
            }
        // (else they are moved behind the branches that follow)
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int f = 0; f < NF; ++f)
                asm volatile("" : "+v"(acc[i][f]));
    };
    // A phase's loads are here when no more than those of the phases behind it are on their way (scales among them: then a wait is longer).
    auto arrive = [&]() {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 3) * C) : "memory");
        lds_barrier();
    };

    issue_scales(0);
#pragma unroll
    for (int d = 0; d < D - 1; ++d)
        issue(d, d);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 2) * C) : "memory");
    lds_barrier();
    read(0, 0, std::integral_constant<int, 0>{}, half[0]);
    int b = 0;
    for (int p = 0; p < phases; ++p) {
        const int next = b == D - 1 ? 0 : b + 1, free = b == 0 ? D - 1 : b - 1;
        each<2 * S>([&](auto hh) {
            constexpr int h = decltype(hh)::value;
            if constexpr (h + 1 < 2 * S) {
                read(p, b, std::integral_constant<int, h + 1>{}, half[(h + 1) & 1]);
            } else {
                arrive();                                       // the next phase; nobody reads the phase before this one any more
                issue(p + D - 1, free);
                if (p % kPhases == 0)
                    issue_scales(p / kPhases + 1);
                read(p + 1, next, std::integral_constant<int, 0>{}, half[0]);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(half[h & 1]);
            __builtin_amdgcn_sched_barrier(0);
        });
        b = next;
    }
    drain_vmem();                                               // (the loads behind the last phase write the LDS)
    __syncthreads();
    if (part) {
        const int ld = tiles_n * BN;
        float* to = part + (int64_t)blockIdx.y * out.m * ld + n0 + wn * NF * 32 + 16 * lh;
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            const int m = m0 + (wm * MF + i) * 32 + li;
            if (m < out.m)
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        *reinterpret_cast<f32x4_t*>(to + (int64_t)m * ld + f * 32 + e) =
                            f32x4_t{acc[i][f][e], acc[i][f][e + 1], acc[i][f][e + 2], acc[i][f][e + 3]};
        }
        return;
    }
    static_assert(leave_bytes(NF) <= D * kBuf, "the operands' place");
    leave<MF, NF>(out, wide, smem + wave * (leave_bytes(NF) / 8), lane, m0 + wm * MF * 32, n0 + wn * NF * 32, acc);
}

// The parts' sums added in order, and what follows them: a thread has one piece of a row.
__global__ __launch_bounds__(256) void w4a8_join_kernel(const float* __restrict__ part, int parts, int ld, bool wide, Out out)
{
    const int piece = out.act == MXFP4_ACT_SWIGLU ? 16 : 8, pieces = (out.n + piece - 1) / piece;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int m = (int)(at / pieces), n = (int)(at % pieces) * piece;
    if (m >= out.m)
        return;
    float z[16];
    f32x4_t sum[4];
    const float* from = part + (int64_t)m * ld + n;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < 2 || piece == 16)
            sum[e] = *reinterpret_cast<const f32x4_t*>(from + 4 * e);
    for (int p = 1; p < parts; ++p) {
        from += (int64_t)out.m * ld;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < 2 || piece == 16)
                sum[e] += *reinterpret_cast<const f32x4_t*>(from + 4 * e);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e)
        z[e] = e < 8 || piece == 16 ? sum[e >> 2][e & 3] : 0.f;
    finish_piece(out, wide, m, n, z);
}

template <int WM, int WN, int MF, int NF, int S, int D>
hipError_t launch(const A8Args& a, int splits, hipStream_t stream)
{
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32;
    static LdsLimit limit;
    const hipError_t raised = limit.raise(reinterpret_cast<const void*>(w4a8_mid_kernel<WM, WN, MF, NF, S, D>), mid_lds(BM, BN, S, D));
    if (raised != hipSuccess)
        return raised;
    const int steps = (a.k + 127) / 128, part_steps = (steps + splits - 1) / splits, parts = (steps + part_steps - 1) / part_steps;
    const int64_t tiles_n = (a.n + BN - 1) / BN, most = max(((int64_t)1 << 22) / (tiles_n * parts), (int64_t)1) * BM;
    for (int64_t at = 0; at < a.m; at += most) {
        const int m = (int)min(most, a.m - at), tiles_m = (m + BM - 1) / BM;
        const Out out = out_of(a, at, m);
        float* part = parts > 1 ? a.part : nullptr;
        w4a8_mid_kernel<WM, WN, MF, NF, S, D><<<dim3((unsigned)(tiles_m * tiles_n), parts), 512, mid_lds(BM, BN, S, D), stream>>>(
            a.x + at * a.k, a.xs + at * (a.k >> 5), a.q, a.s, a.k, tiles_m, (int)tiles_n, part_steps, part, wide_rows(a), out);
        if (part) {
            const int piece = a.epi.act == MXFP4_ACT_SWIGLU ? 16 : 8;
            const int64_t threads = (int64_t)m * ((a.n + piece - 1) / piece);
            w4a8_join_kernel<<<dim3((unsigned)((threads + 255) / 256)), 256, 0, stream>>>(part, parts, (int)tiles_n * BN, wide_rows(a), out);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_mid(const A8Args& a, int shape, int splits, hipStream_t stream)
{
    switch (shape) {
    case 1:
        return launch<2, 4, 1, 1, 2, 4>(a, splits, stream);
    case 2:
        return launch<2, 4, 2, 1, 1, 5>(a, splits, stream);
    case 4:
        return launch<4, 2, 1, 1, 1, 5>(a, splits, stream);
    case 5:
        return launch<1, 8, 1, 1, 1, 5>(a, splits, stream);
    case 6:
        return launch<2, 4, 2, 2, 1, 3>(a, splits, stream);
    case 7:
        return launch<2, 4, 1, 1, 1, 6>(a, splits, stream);
    default:
        return launch<2, 4, 1, 1, 2, 4>(a, splits, stream);
    }
}

}  // namespace a8
}  // namespace mxfp4
