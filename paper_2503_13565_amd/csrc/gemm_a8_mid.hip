// The product of 8-bit rows with MXFP4 weights for some tens to some hundreds of rows (gemm_a8.hip: fewer, gemm_a8_block.hip: more).
//
// The instructions and the LDS layout of gemm_a8_block.hip in smaller blocks, of which one alone does not fill its compute unit's time: what bounds
// them is how long a step takes from its arrival to its sums.  So the eight waves are WM x WN x WK: WK of them share the steps of a phase, each on a
// step of its own (their sums meet in the LDS at the end, in order), which halves and quarters what the waves read of each other's rows, and the barriers.
// The loads of a phase leave as soon as its buffer has been read, D - 1 phases ahead, and a phase waits for its own loads only.  That takes scales
// that no wait of the compiler's stands in front of: they come into the LDS by direct loads too, sixteen steps at a time (64 bytes a row and up to 16
// around them: a row of K / 32 bytes may start anywhere, a load starts at a dword; 80 bytes from row to row put two lanes on a bank), and a lane reads a
// step's four in two dwords and moves its own to the bytes that the instruction names.
// Bound by the walk of each block, and for larger ones by the lines that a unit gets from beyond its die's cache (80 to 90 bytes a ns).  77 rows x
// 4096 x 11008 take 14.4 us in 192 blocks of 32 x 64, 16.4 where the weights are in no cache (25 MB, 3.8 us at the rate of a kernel that only reads): start, first
// phase and end are 4.9, and in the 21 phases behind it loads, scales and matrix instructions wait for each other in part (each left out alone saved 3.8, 2.5 and
// 3.1 of the 15.8 before the loads went out in quarters); 42 % of the LDS's active cycles are conflicts.  No gain: four phases in the
// LDS, eight waves along K, sixteen waves; K cut across workgroups with a second kernel that adds was slower (17 to 18 us).
#include "block_out.h"
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

template <int WM, int WN, int WK, int MF, int NF, int D>
__global__ __launch_bounds__(512, 2) void w4a8_mid_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xs,
                                                          const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, int k, int tiles_m,
                                                          int tiles_n, bool wide, Out out)
{
    static_assert(WM * WN * WK == 8, "eight waves");
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32, S = WK;
    constexpr int kBuf = mid_buffer(BM, BN, S), kX = BM * S / 8, kUnits = phase_units(BM, BN, S), C = (kUnits + 7) / 8;
    constexpr int kSx = scale_units(BM), kScaleUnits = kSx + scale_units(BN), kPhases = kScaleSteps / S;
    static_assert(mid_lds(BM, BN, S, D) <= 160 * 1024 && D <= kPhases, "the LDS; scales arrive before their steps");
    extern __shared__ __align__(16) uint8_t smem[];
    const int lane = threadIdx.x & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / (WN * WK), wn = wave / WK % WN, wk = wave % WK;
    const int nblk = k >> 5, steps = (k + 127) >> 7, phases = (steps + S - 1) / S;
    const int at = block_on_die(tiles_m * tiles_n, blockIdx.x), m0 = at % tiles_m * BM, n0 = at / tiles_m * BN;
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
        const int piece = (of_x ? u : u - kX) * 64 + lane;
        chunk[c] = of_x ? piece_chunk(piece, S * 8) : piece_chunk(piece, S * 4);
        off[c] = u >= kUnits ? kOob : of_x ? piece_offset(piece, S * 8, rows, k) : piece_offset(piece, S * 4, cols, k >> 1);
    }
    // A quarter of a phase's loads (past K's end: zeros, so that the loads of a phase are as many).
    auto issue = [&](int p, int b, auto quarter) {
        const int t = p * S;
#pragma unroll
        for (int c = decltype(quarter)::value; c < C; c += 4) {
            const int u = c * 8 + wave;
            if (u < kX)
                direct(lds_at + b * kBuf + u * 1024, off[c] | past((k >> 4) - 1, phase_chunk(t, 128) + chunk[c]), rx, phase_from(t, steps, 128));
            else
                direct(lds_at + (u < kUnits ? b * kBuf + u * 1024 : D * kBuf + 2048 * kScaleUnits), off[c] | past(nblk - 1, phase_chunk(t, 64) + chunk[c]),
                       rq, phase_from(t, steps, 64));
        }
    };
    auto issue_scales = [&](int part16) {                       // of the sixteen steps from 16 part16 on
#pragma unroll
        for (int c = 0; c < (kScaleUnits + 7) / 8; ++c) {
            const int u = c * 8 + wave;
            if (u < kScaleUnits) {
                const bool of_x = u < kSx;
                const int piece = (of_x ? u : u - kSx) * 64 + lane, row = piece / (kScaleRow / 16), in = piece % (kScaleRow / 16) * 16;
                const uint32_t to = lds_at + D * kBuf + ((part16 & 1) * kScaleUnits + u) * 1024;
                const int o = (((row * nblk + part16 * (4 * kScaleSteps)) & ~3) + in) | past((of_x ? rows : cols) - 1, row);
                if (of_x)
                    direct(to, o, rxs, 0);
                else
                    direct(to, o, rs, 0);
            }
        }
    };

    // The operands of one half of this wave's step of a phase; the scales are of both halves: bytes 0 and 2.
    struct Half {
        u32x4_t x[MF][2], w[NF];
    } half[2];
    uint32_t xs_of[MF], ws_of[NF];
    const int wrow = 16 * (li >> 2 & 1) + 4 * (li >> 3) + (li & 3);
    const int x_row = wm * MF * 32 + li, w_row = wn * NF * 32 + wrow;
    const int x_read = x_row * (S * 128) + ((8 * wk + lh) ^ turn(x_row, S * 8)) * 16;
    const int w_read = kX * 1024 + w_row * (S * 64) + ((4 * wk + lh) ^ turn(w_row, S * 4)) * 16;
    int xs_first[MF], ws_first[NF];                             // where the row's first byte is in its dword
#pragma unroll
    for (int f = 0; f < MF; ++f)
        xs_first[f] = ((x_row + f * 32) * nblk) & 3;
#pragma unroll
    for (int f = 0; f < NF; ++f)
        ws_first[f] = ((w_row + f * 32) * nblk) & 3;
    const uint8_t *xs_read = smem + D * kBuf + x_row * kScaleRow, *ws_read = smem + D * kBuf + kSx * 1024 + w_row * kScaleRow;
    // A phase's dwords may leave for registers beside the instructions of the phase before, which still need theirs, and are moved behind these.
    uint2 xs_raw[MF], ws_raw[NF];
    auto fetch_scales = [&](int p) {
        const int in = ((p / kPhases) & 1) * (kScaleUnits * 1024) + ((p % kPhases) * S + wk) * 4;
        const auto two = [&](const uint8_t* row) {
            const uint32_t* at = reinterpret_cast<const uint32_t*>(row + in);
            return make_uint2(at[0], at[1]);
        };
#pragma unroll
        for (int f = 0; f < MF; ++f)
            xs_raw[f] = two(xs_read + f * (32 * kScaleRow));
#pragma unroll
        for (int f = 0; f < NF; ++f)
            ws_raw[f] = two(ws_read + f * (32 * kScaleRow));
    };
    auto take_scales = [&](int p) {
        const int have = nblk - 4 * (p * S + wk);               // blocks of this step; behind the last, the bytes are another row's
        const uint32_t keep = have >= 4 ? 0xFFFFFFFFu : have <= 0 ? 0u : (1u << (8 * have)) - 1u;
        const auto bytes = [&](const uint2& raw, int first) { return (__builtin_amdgcn_alignbyte(raw.y, raw.x, first) & keep) >> (8 * lh); };
#pragma unroll
        for (int f = 0; f < MF; ++f)
            xs_of[f] = bytes(xs_raw[f], xs_first[f]);
#pragma unroll
        for (int f = 0; f < NF; ++f)
            ws_of[f] = bytes(ws_raw[f], ws_first[f]);
    };
    auto read = [&](int b, int kh, Half& h) {                   // half kh of the phase in buffer b
        const uint8_t* buf = smem + b * kBuf;
#pragma unroll
        for (int f = 0; f < NF; ++f)
            h.w[f] = *reinterpret_cast<const u32x4_t*>(buf + (w_read ^ (kh * 32)) + f * (32 * S * 64));
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            h.x[f][0] = *reinterpret_cast<const u32x4_t*>(buf + (x_read ^ (kh * 64)) + f * (32 * S * 128));
            h.x[f][1] = *reinterpret_cast<const u32x4_t*>(buf + (x_read ^ (kh * 64 + 32)) + f * (32 * S * 128));
        }
    };
    f32x16_t acc[MF][NF] = {};
    auto multiply = [&](const Half& h, auto kh) {
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                const u32x4_t w = h.w[f], x0 = h.x[i][0], x1 = h.x[i][1];
                const i32x8_t A = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
                const i32x8_t B = {(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
                acc[i][f] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, acc[i][f], 4, 0, 2 * decltype(kh)::value, (int)ws_of[f],
                                                                           2 * decltype(kh)::value, (int)xs_of[i]);
                settle(acc[i][f]);                              // (else they are moved behind the branches that follow)
            }
    };

    issue_scales(0);
#pragma unroll
    for (int d = 0; d < D; ++d)
        each<4>([&](auto quarter) { issue(d, d, quarter); });
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * C) : "memory");
    lds_barrier();
    issue_scales(1);
    fetch_scales(0);
    take_scales(0);
    read(0, 0, half[0]);
    int b = 0, before = D - 1;
    // Where two phases are on their way, the loads of another go out a quarter at a time between the reads and the instructions: all at once behind
    // the barrier, the waves of all SIMDs wait for the way out (16 cycles a load) before they read (128 x 4096 x 4096 10.0 us, 9.7 so).  Where it is one,
    // every cycle that they leave earlier counts (128 x 22016 x 4096 23.9 us, 27.3 in quarters), and so does a register (25.7 with the scales fetched early).
    constexpr bool kSpread = D > 2;
    constexpr std::integral_constant<int, 0> first;
    constexpr std::integral_constant<int, 1> second;
    constexpr std::integral_constant<int, 2> third;
    constexpr std::integral_constant<int, 3> fourth;
    for (int p = 0; p < phases; ++p) {
        const int next = b == D - 1 ? 0 : b + 1;
        read(b, 1, half[1]);
        if (kSpread && p)
            issue(p - 1 + D, before, third);
        __builtin_amdgcn_sched_barrier(0);
        multiply(half[0], first);
        __builtin_amdgcn_sched_barrier(0);
        if (kSpread && p)
            issue(p - 1 + D, before, fourth);
        // The next phase is here when no more loads than those of the phases behind it are on their way (with scales among them, a wait is longer); this one's
        // buffer is free when every wave has its second half in registers.
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 2) * C) : "memory");
        lds_barrier();
        if constexpr (kSpread)
            issue(p + D, b, first);
        else
            each<4>([&](auto quarter) { issue(p + D, b, quarter); });
        if (p % kPhases == kPhases - 1)
            issue_scales(p / kPhases + 2);                      // (of the sixteen steps behind the next: into the place of those that end here)
        if (kSpread)
            fetch_scales(p + 1);
        read(next, 0, half[0]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(half[1], second);
        if (kSpread)
            issue(p + D, b, second);
        if (!kSpread)
            fetch_scales(p + 1);
        take_scales(p + 1);
        __builtin_amdgcn_sched_barrier(0);
        before = b;
        b = next;
    }
    drain_vmem();                                               // (the loads behind the last phase write the LDS)
    __syncthreads();

    // Out through the LDS: the sums of the waves that shared the steps side by side, and every thread adds those of its pieces of rows.
    constexpr int kLd = BN + 4;
    static_assert(WK * BM * kLd * 4 <= mid_lds(BM, BN, S, D), "the operands' place");
    float* tile = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4_t*>(tile + (wk * BM + x_row + i * 32) * kLd + (wn * NF + f) * 32 + 16 * lh + e) =
                    f32x4_t{acc[i][f][e], acc[i][f][e + 1], acc[i][f][e + 2], acc[i][f][e + 3]};
    __syncthreads();
    const int piece = out.act == MXFP4_ACT_SWIGLU ? 16 : 8, pieces = BN / piece;
    for (int at = threadIdx.x; at < BM * pieces; at += 512) {
        const int row = at / pieces, n = at % pieces * piece;
        if (m0 + row < out.m && n0 + n < out.n)
            finish_piece<WK>(out, wide, m0 + row, n0 + n, tile + row * kLd + n, BM * kLd);
    }
}

template <int WM, int WN, int WK, int MF, int NF, int D>
hipError_t launch(const A8Args& a, hipStream_t stream)
{
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32;
    static LdsLimit limit;
    const hipError_t raised = limit.raise(reinterpret_cast<const void*>(w4a8_mid_kernel<WM, WN, WK, MF, NF, D>), mid_lds(BM, BN, WK, D));
    if (raised != hipSuccess)
        return raised;
    const int64_t tiles_n = (a.n + BN - 1) / BN, most = max(((int64_t)1 << 22) / tiles_n, (int64_t)1) * BM;
    for (int64_t at = 0; at < a.m; at += most) {
        const int m = (int)min(most, a.m - at), tiles_m = (m + BM - 1) / BM;
        w4a8_mid_kernel<WM, WN, WK, MF, NF, D><<<dim3((unsigned)(tiles_m * tiles_n)), 512, mid_lds(BM, BN, WK, D), stream>>>(
            a.x + at * a.k, a.xs + at * (a.k >> 5), a.q, a.s, a.k, tiles_m, (int)tiles_n, wide_rows(a), out_of(a, at, m));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_mid(const A8Args& a, Shape shape, hipStream_t stream)
{
    switch (shape) {
    case kMid32x64:
        return launch<1, 2, 4, 1, 1, 2>(a, stream);
    case kMid32x64Deep:
        return launch<1, 2, 4, 1, 1, 3>(a, stream);
    case kMid64x128:
        return launch<2, 2, 2, 1, 2, 3>(a, stream);
    default:
        return launch<2, 2, 2, 2, 2, 2>(a, stream);
    }
}

}  // namespace a8
}  // namespace mxfp4
