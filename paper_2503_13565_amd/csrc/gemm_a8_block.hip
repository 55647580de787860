// The product of 8-bit rows with MXFP4 weights for many rows (gemm_a8.hip has the few).
//
// A workgroup of eight waves computes BM x BN outputs and walks K in steps of 128.  Both operands of a step lie in the LDS as they lie in
// memory, brought there by loads that write it directly, a step and more ahead of their use; three buffers, one barrier a step.  A wave
// computes MF x NF tiles of 32 x 32 with v_mfma_scale_f32_32x32x64_f8f6f4, the weights as its rows: for one half of a step lane
// i + 32 h holds, of row i, 16 bytes of weights (block h), of x 16 bytes from 16 h on and 16 from 32 + 16 h on.  The reads of a half go
// out beside the instructions of the half before it, across the barrier too.
//
//   - Weight row i of a tile's operand is row 16 (i / 4 % 2) + 4 (i / 8) + i % 4 of the tile, so that a lane's 16 sums of a tile are 16
//     outputs side by side.
//   - Chunk c (16 bytes) of x's row r lies at c ^ (r / 2 % 8) of the row's eight, of a weight row at c ^ (r / 4 % 4) of its four: the sixteen
//     lanes that a turn of the LDS serves find sixteen different places.
//   - Scale bytes come through registers four steps at a time (16 bytes a row, at any address, as K / 32 may be any number) and are laid out
//     by position: [step][block][wave row][i][tile], so that one read gives a lane the bytes of all its tiles, which the
//     instruction takes by number.  Blocks past K get zero bytes, as their codes load as zeros.
//
// 4003 rows x 22016 x 4096 with the gate: 311 to 327 us by the card's clock, 2.2 to 2.3 PFLOP/s (a loop of the bare instruction: 4.5, of random
// numbers).  The matrix units are busy for 62 % of the cycles, at a clock that their power draw lowers (all zeros: 9 % less time); the LDS for a third,
// without conflicts; waves wait for 39 % of their time.  That is in blocks of 128 x 256, two on a unit, which fill the last round better than those of
// 256 x 256 with their 2/3 of the traffic; alone they take the same time.  In 256 x 256, four waves of twice the tile read 40 % less from the
// LDS and were slower (351 us, 337 with eight then), and so were loads two steps ahead (326, 319).
#include "block_out.h"
#include "gemm_a8.h"

namespace mxfp4 {
namespace a8 {

namespace {

constexpr int lds_buffer(int bm, int bn) { return bm * 128 + bn * 64; }
constexpr int lds_bytes(int bm, int bn, int d) { return d * lds_buffer(bm, bn) + 2 * 16 * (bm + bn); }

// 16 scale bytes of a row from block `at` on; zeros past its end.  No byte outside the row is read.
__device__ __forceinline__ u32x4_t scale_bytes(const uint8_t* row, int at, int nblk)
{
    u32x4_t v = {0, 0, 0, 0};
    if (at + 16 <= nblk) {
        __builtin_memcpy(&v, row + at, 16);
    } else if (nblk >= 16) {                                    // the row's last 16 bytes, moved down
        __builtin_memcpy(&v, row + nblk - 16, 16);
        const int gone = 8 * (at + 16 - nblk);                  // bits, 8 .. 120
        unsigned __int128 w;
        __builtin_memcpy(&w, &v, 16);
        w >>= gone;
        __builtin_memcpy(&v, &w, 16);
    } else {
        for (int i = 0; i < nblk; ++i)                          // (one group: at is 0)
            v[i >> 2] |= (uint32_t)row[i] << (8 * (i & 3));
    }
    return v;
}

template <int WM, int WN, int MF, int NF, int D>
__global__ __launch_bounds__(WM * WN * 64, D == 2 ? 4 : WM * WN / 4) void w4a8_block_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xs,
                                                            const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, int k, int tiles_m,
                                                            int tiles_n, bool wide, Out out)
{
    constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32, CX = BM / 8 / kWaves, CW = BN / 16 / kWaves, kRows = (BM + BN + kThreads - 1) / kThreads;
    constexpr int kBuf = lds_buffer(BM, BN), kScales = 16 * (BM + BN);
    static_assert(lds_bytes(BM, BN, D) <= (D == 2 ? 80 : 160) * 1024 && CX * 8 * kWaves == BM && CW * 16 * kWaves == BN && (D == 2 || (kRows * kThreads == BM + BN && BM == BN)),
                  "the LDS; whole instructions a wave; whole rows of scales a thread");
    extern __shared__ __align__(16) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int nblk = k >> 5, steps = (k + 127) >> 7;
    const bool ragged = (k & 127) != 0;

    // The 32 blocks that a die runs at once are four rows of blocks by eight columns: they read 4 x 32 and 8 x 16 KiB a step through the die's L2.
    const int at = block_on_die(tiles_m * tiles_n, blockIdx.x), band = at / (4 * tiles_n), band_m = min(4, tiles_m - 4 * band), in_band = at - band * 4 * tiles_n;
    const int m0 = (4 * band + in_band % band_m) * BM, n0 = in_band / band_m * BN;
    const int rows = min(BM, out.m - m0), cols = min(BN, out.n - n0);

    const u32x4_t rx = words(x + (int64_t)m0 * k, rows * k), rq = words(q + (int64_t)n0 * (k >> 1), cols * (k >> 1));
    const uint32_t lds_at = lds_address(smem);

    // Load i of wave w fills KiB kWaves i + w of a step's x (8 rows of 128 bytes) or weights (16 rows of 64).
    int x_off[CX], x_chunk[CX], w_off[CW], w_chunk[CW];
#pragma unroll
    for (int i = 0; i < CX; ++i) {
        const int row = (i * kWaves + wave) * 8 + (lane >> 3);
        x_chunk[i] = (lane & 7) ^ (row >> 1 & 7);
        x_off[i] = (row * k + x_chunk[i] * 16) | past(rows - 1, row);
    }
#pragma unroll
    for (int i = 0; i < CW; ++i) {
        const int row = (i * kWaves + wave) * 16 + (lane >> 2);
        w_chunk[i] = (lane & 3) ^ (row >> 2 & 3);
        w_off[i] = (row * (k >> 1) + w_chunk[i] * 16) | past(cols - 1, row);
    }
    auto issue = [&](int T, int b) {
        const uint32_t to = lds_at + b * kBuf + wave * 1024;
        const bool tail = ragged && T == steps - 1;
#pragma unroll
        for (int i = 0; i < CX; ++i)
            direct(to + i * (kWaves * 1024), x_off[i] | (tail ? past((k >> 4) - 1, T * 8 + x_chunk[i]) : 0), rx, T * 128);
#pragma unroll
        for (int i = 0; i < CW; ++i)
            direct(to + BM * 128 + i * (kWaves * 1024), w_off[i] | (tail ? past(nblk - 1, T * 4 + w_chunk[i]) : 0), rq, T * 64);
    };

    // This thread's rows of scales and where their bytes go (for step t and block b: + (4 t + b) * rows of the operand).
    uint8_t* scales = smem + D * kBuf;
    const uint8_t* s_from[kRows];
    int s_to[kRows];
    bool s_live[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const bool of_x = i * kThreads + tid < BM;
        const int row = i * kThreads + tid - (of_x ? 0 : BM);
        s_live[i] = i * kThreads + tid < BM + BN && row < (of_x ? rows : cols);
        s_from[i] = (of_x ? xs + (int64_t)m0 * nblk : s + (int64_t)n0 * nblk) + (int64_t)(s_live[i] ? row : 0) * nblk;
        const int tiles = of_x ? MF : NF, r = row & 31;
        const int at32 = of_x ? r : 8 * (r >> 2 & 3) + 4 * (r >> 4) + (r & 3);
        s_to[i] = (of_x ? 0 : 16 * BM) + (row / (32 * tiles) * 32 + at32) * tiles + row / 32 % tiles;
    }
    u32x4_t sv[kRows] = {};
    auto load_scales = [&](int group) {
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (s_live[i] && group * 16 < nblk)
                sv[i] = scale_bytes(s_from[i], group * 16, nblk);
    };
    auto store_scales = [&](int group) {
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (kRows * kThreads == BM + BN || i * kThreads + tid < BM + BN)
#pragma unroll
            for (int b = 0; b < 16; ++b)
                scales[(group & 1) * kScales + s_to[i] + b * (BM == BN || i * kThreads + tid < BM ? BM : BN)] = (uint8_t)(sv[i][b >> 2] >> (8 * (b & 3)));
    };

    // The operands of half a step.
    struct Half {
        u32x4_t x[MF][2], w[NF];
        uint32_t xs, ws;
    } half[2];
    const int a = li >> 3, wrow = 16 * (li >> 2 & 1) + 4 * a + (li & 3);
    const int x_read = (wm * MF * 32 + li) * 128 + (lh ^ (li >> 1 & 7)) * 16;
    const int w_read = BM * 128 + (wn * NF * 32 + wrow) * 64 + (lh ^ a) * 16;
    const int xs_read = (lh * WM * 32 + wm * 32 + li) * MF, ws_read = 16 * BM + (lh * WN * 32 + wn * 32 + li) * NF;
    // The reads of half kh of step T, which lies in buffer b, one by one: scales, weights, x.
    constexpr int kReads = 1 + NF + 2 * MF;
    auto read = [&](int T, int b, auto kh, Half& h, auto which) {
        constexpr int at = decltype(which)::value;
        const uint8_t* buf = smem + b * kBuf;
        if constexpr (at == 0) {
            const uint8_t* sc = scales + (T >> 2 & 1) * kScales;
            const int part = (T & 3) * 4 + 2 * kh;
            auto bytes = [](const uint8_t* p, auto n) -> uint32_t {
                if constexpr (n == 4)
                    return *reinterpret_cast<const uint32_t*>(p);
                else if constexpr (n == 2)
                    return *reinterpret_cast<const uint16_t*>(p);
                else
                    return *p;
            };
            h.xs = bytes(sc + xs_read + part * BM, std::integral_constant<int, MF>{});
            h.ws = bytes(sc + ws_read + part * BN, std::integral_constant<int, NF>{});
        } else if constexpr (at <= NF) {
            h.w[at - 1] = *reinterpret_cast<const u32x4_t*>(buf + (w_read ^ (kh * 32)) + (at - 1) * 2048);
        } else if constexpr (at < kReads) {
            constexpr int f = (at - 1 - NF) / 2, hi = (at - 1 - NF) % 2;
            h.x[f][hi] = *reinterpret_cast<const u32x4_t*>(buf + (x_read ^ (kh * 64 + hi * 32)) + f * 4096);
        }
    };
    f32x16_t acc[MF][NF] = {};
    // The instructions of a half, and between(j) behind instruction j: an instruction holds the matrix pipe for 64 cycles, in which what is between
    // them leaves for free; in front of them all, the reads of eight waves keep the pipe waiting for 640 (the prompt 345 us).
    auto multiply = [&](const Half& h, auto between) {
        each<MF>([&](auto i) {
            each<NF>([&](auto f) {
                const u32x4_t w = h.w[f], x0 = h.x[i][0], x1 = h.x[i][1];
                const i32x8_t A = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
                const i32x8_t B = {(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
                acc[i][f] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, acc[i][f], 4, 0, decltype(f)::value, (int)h.ws,
                                                                           decltype(i)::value, (int)h.xs);
                settle(acc[i][f]);
                if constexpr (D > 2)
                    __builtin_amdgcn_sched_barrier(0);
                between(std::integral_constant<int, decltype(i)::value * NF + decltype(f)::value>{});
                if constexpr (D > 2)
                    __builtin_amdgcn_sched_barrier(0);
            });
        });
    };
    constexpr int kEach = (kReads + MF * NF - 2) / (MF * NF - 1);       // reads behind an instruction
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};

    load_scales(0);
    issue(0, 0);
    if constexpr (D == 2) {
        store_scales(0);
        load_scales(1);
        for (int T = 0; T < steps; ++T) {
            drain_vmem();                                       // this step's loads, which left a step ago
            if ((T & 3) == 3)
                store_scales((T >> 2) + 1);
            lds_barrier();
            if (T + 1 < steps)
                issue(T + 1, (T + 1) & 1);
            if ((T & 3) == 3)
                load_scales((T >> 2) + 2);
            each<kReads>([&](auto r) { read(T, T & 1, first, half[0], r); });
            multiply(half[0], [&](auto) {});
            each<kReads>([&](auto r) { read(T, T & 1, second, half[0], r); });
            multiply(half[0], [&](auto) {});
        }
        __syncthreads();
        leave<MF, NF>(out, wide, smem + wave * (leave_bytes(NF) / 8), lane, m0 + wm * MF * 32, n0 + wn * NF * 32, acc);
        return;
    }
    if (steps > 1)
        issue(1, 1);
    store_scales(0);
    drain_vmem();
    lds_barrier();
    load_scales(1);
    each<kReads>([&](auto r) { read(0, 0, first, half[0], r); });
    int b = 0;                                                  // the step's buffer
    // (Without a condition around what changes registers: behind the last step a buffer is read that nothing uses.)
    for (int T = 0; T < steps; ++T) {
        const int next = b == 2 ? 0 : b + 1, free = next == 2 ? 0 : next + 1;
        multiply(half[0], [&](auto j) {
            each<kEach>([&](auto e) { read(T, b, second, half[1], std::integral_constant<int, decltype(j)::value * kEach + decltype(e)::value>{}); });
        });
        multiply(half[1], [&](auto j) {
            constexpr int at = decltype(j)::value;
            if constexpr (at == 0) {
                drain_vmem();                                   // the next step's loads, which left a step ago
                if ((T & 3) == 2)
                    store_scales((T >> 2) + 1);
                lds_barrier();
                if (T + 2 < steps)
                    issue(T + 2, free);
                if ((T & 3) == 3)
                    load_scales((T >> 2) + 2);
            } else {
                each<kEach>([&](auto e) { read(T + 1, next, first, half[0], std::integral_constant<int, (at - 1) * kEach + decltype(e)::value>{}); });
            }
        });
        b = next;
    }
    static_assert(leave_bytes(NF) / 8 * kWaves <= lds_bytes(BM, BN, D), "the operands' place");
    __syncthreads();
    leave<MF, NF>(out, wide, smem + wave * (leave_bytes(NF) / 8), lane, m0 + wm * MF * 32, n0 + wn * NF * 32, acc);
}

template <int WM, int WN, int MF, int NF, int D>
hipError_t launch(const A8Args& a, hipStream_t stream)
{
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32;
    static LdsLimit limit;
    const hipError_t raised = limit.raise(reinterpret_cast<const void*>(w4a8_block_kernel<WM, WN, MF, NF, D>), lds_bytes(BM, BN, D));
    if (raised != hipSuccess)
        return raised;
    const int64_t tiles_n = (a.n + BN - 1) / BN, most = max(((int64_t)1 << 22) / tiles_n, (int64_t)1) * BM;
    for (int64_t at = 0; at < a.m; at += most) {
        const int m = (int)min(most, a.m - at), tiles_m = (m + BM - 1) / BM;
        w4a8_block_kernel<WM, WN, MF, NF, D><<<dim3((unsigned)(tiles_m * tiles_n)), WM * WN * 64, lds_bytes(BM, BN, D), stream>>>(
            a.x + at * a.k, a.xs + at * (a.k >> 5), a.q, a.s, a.k, tiles_m, (int)tiles_n, wide_rows(a), out_of(a, at, m));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_block(const A8Args& a, Shape shape, hipStream_t stream)
{
    return shape == kBlock128x256 ? launch<2, 4, 2, 2, 2>(a, stream) : launch<2, 4, 4, 2, 3>(a, stream);
}

}  // namespace a8
}  // namespace mxfp4
