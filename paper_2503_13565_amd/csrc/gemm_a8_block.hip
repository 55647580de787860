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
#include <utility>

#include "gemm_a8.h"

namespace mxfp4 {
namespace a8 {

namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;

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

constexpr int lds_buffer(int bm, int bn) { return bm * 128 + bn * 64; }
constexpr int lds_bytes(int bm, int bn) { return 3 * lds_buffer(bm, bn) + 2 * 16 * (bm + bn); }

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

template <int WM, int WN, int MF, int NF>
__global__ __launch_bounds__(512, 2) void w4a8_block_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ xs,
                                                            const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, int k, int tiles_m,
                                                            int tiles_n, bool wide, Out out)
{
    static_assert(WM * WN == 8, "eight waves");
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32, CX = BM / 64, CW = BN / 128;
    constexpr int kBuf = lds_buffer(BM, BN), kScales = 16 * (BM + BN);
    static_assert(lds_bytes(BM, BN) <= 160 * 1024 && BN % 128 == 0 && BM + BN <= 512, "the LDS; whole instructions a wave; a row a thread");
    extern __shared__ __align__(16) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;
    const int nblk = k >> 5, steps = (k + 127) >> 7;
    const bool ragged = (k & 127) != 0;

    // Blocks that run together on a die share rows of x and of the weights: columns of up to eight blocks of rows.
    const int at = blockIdx.x, band = at / (8 * tiles_n), band_m = min(8, tiles_m - 8 * band), in_band = at - band * 8 * tiles_n;
    const int m0 = (8 * band + in_band % band_m) * BM, n0 = in_band / band_m * BN;
    const int rows = min(BM, out.m - m0), cols = min(BN, out.n - n0);

    auto words = [](const uint8_t* p, int bytes) {
        auto uniform = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
        const uint64_t a = reinterpret_cast<uint64_t>(p);
        return u32x4_t{uniform((uint32_t)a), uniform((uint32_t)(a >> 32) & 0xFFFFu), uniform((uint32_t)bytes), 0x00020000u};
    };
    const u32x4_t rx = words(x + (int64_t)m0 * k, rows * k), rq = words(q + (int64_t)n0 * (k >> 1), cols * (k >> 1));
    const uint32_t lds_at = (uint32_t)reinterpret_cast<uint64_t>((__attribute__((address_space(3))) uint8_t*)smem);

    // Load i of wave w fills KiB 8 i + w of a step's x (8 rows of 128 bytes) or weights (16 rows of 64).
    int x_off[CX], x_chunk[CX], w_off[CW], w_chunk[CW];
#pragma unroll
    for (int i = 0; i < CX; ++i) {
        const int row = (i * 8 + wave) * 8 + (lane >> 3);
        x_chunk[i] = (lane & 7) ^ (row >> 1 & 7);
        x_off[i] = (row * k + x_chunk[i] * 16) | past(rows - 1, row);
    }
#pragma unroll
    for (int i = 0; i < CW; ++i) {
        const int row = (i * 8 + wave) * 16 + (lane >> 2);
        w_chunk[i] = (lane & 3) ^ (row >> 2 & 3);
        w_off[i] = (row * (k >> 1) + w_chunk[i] * 16) | past(cols - 1, row);
    }
    // m0: where in the LDS lane 0's bytes go.  The load reads scalar registers that a vector instruction may have written just in front:
    // five wait states, which the compiler does not count into assembly.
    auto direct = [](uint32_t to, int off, const u32x4_t& r, int from) {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(off), "s"(r), "s"(from)
                     : "memory", "m0");
    };
    auto issue = [&](int T, int b) {
        const uint32_t to = lds_at + b * kBuf + wave * 1024;
        const bool tail = ragged && T == steps - 1;
#pragma unroll
        for (int i = 0; i < CX; ++i)
            direct(to + i * 8192, x_off[i] | (tail ? past((k >> 4) - 1, T * 8 + x_chunk[i]) : 0), rx, T * 128);
#pragma unroll
        for (int i = 0; i < CW; ++i)
            direct(to + BM * 128 + i * 8192, w_off[i] | (tail ? past(nblk - 1, T * 4 + w_chunk[i]) : 0), rq, T * 64);
    };

    // This thread's row of scales and where its bytes go (for step t and block b: + (4 t + b) * 32 * tiles of a row or column of waves).
    const bool of_x = tid < BM;
    const int s_row = of_x ? tid : tid - BM;
    const bool s_live = of_x ? s_row < rows : s_row < cols;
    const uint8_t* s_from = (of_x ? xs + (int64_t)m0 * nblk : s + (int64_t)n0 * nblk) + (int64_t)(s_live ? s_row : 0) * nblk;
    int s_to, s_step;
    if (of_x) {
        const int w = s_row / (32 * MF), f = s_row / 32 % MF, i = s_row & 31;
        s_to = (w * 32 + i) * MF + f;
        s_step = BM;
    } else {
        const int w = s_row / (32 * NF), f = s_row / 32 % NF, n = s_row & 31, i = 8 * (n >> 2 & 3) + 4 * (n >> 4) + (n & 3);
        s_to = 16 * BM + (w * 32 + i) * NF + f;
        s_step = BN;
    }
    uint8_t* scales = smem + 3 * kBuf;
    u32x4_t sv = {0, 0, 0, 0};
    auto load_scales = [&](int group) {
        if (tid < BM + BN && s_live && group * 16 < nblk)
            sv = scale_bytes(s_from, group * 16, nblk);
    };
    auto store_scales = [&](int group) {
        uint8_t* to = scales + (group & 1) * kScales + s_to;
        if (tid < BM + BN)
#pragma unroll
            for (int b = 0; b < 16; ++b)
                to[b * s_step] = (uint8_t)(sv[b >> 2] >> (8 * (b & 3)));
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
    auto read = [&](int T, int b, auto kh, Half& h) {
        const uint8_t* buf = smem + b * kBuf;
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
#pragma unroll
        for (int f = 0; f < NF; ++f)
            h.w[f] = *reinterpret_cast<const u32x4_t*>(buf + (w_read ^ (kh * 32)) + f * 2048);
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            h.x[f][0] = *reinterpret_cast<const u32x4_t*>(buf + (x_read ^ (kh * 64)) + f * 4096);
            h.x[f][1] = *reinterpret_cast<const u32x4_t*>(buf + (x_read ^ (kh * 64 + 32)) + f * 4096);
        }
    };
    f32x16_t acc[MF][NF] = {};
    auto multiply = [&](const Half& h) {
        each<MF>([&](auto i) {
            each<NF>([&](auto f) {
                const u32x4_t w = h.w[f], x0 = h.x[i][0], x1 = h.x[i][1];
                const i32x8_t A = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
                const i32x8_t B = {(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
                acc[i][f] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(A, B, acc[i][f], 4, 0, decltype(f)::value, (int)h.ws,
                                                                           decltype(i)::value, (int)h.xs);
            });
        });
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};

    load_scales(0);
    issue(0, 0);
    if (steps > 1)
        issue(1, 1);
    store_scales(0);
    drain_vmem();
    lds_barrier();
    load_scales(1);
    read(0, 0, first, half[0]);
    int b = 0;                                                  // the step's buffer
    // (Without a condition around what changes registers: behind the last step a buffer is read that nothing uses.)
    for (int T = 0; T < steps; ++T) {
        const int next = b == 2 ? 0 : b + 1, free = next == 2 ? 0 : next + 1;
        read(T, b, second, half[1]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(half[0]);
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int f = 0; f < NF; ++f)
                asm volatile("" : "+v"(acc[i][f]));             // (else they are moved behind the branches below)
        __builtin_amdgcn_sched_barrier(0);
        drain_vmem();                                           // the next step's loads, which left a step ago
        if ((T & 3) == 2)
            store_scales((T >> 2) + 1);
        lds_barrier();
        if (T + 2 < steps)
            issue(T + 2, free);
        if ((T & 3) == 3)
            load_scales((T >> 2) + 2);
        read(T + 1, next, first, half[0]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(half[1]);
        __builtin_amdgcn_sched_barrier(0);
        b = next;
    }

    // Out through the LDS, 32 rows at a time, so that whole pieces of rows are stored.  Each wave has a part of its own.
    constexpr int kCols = 32 * NF, kStride = kCols + 4;
    static_assert(8 * 32 * kStride * 4 <= 3 * kBuf, "the operands' place");
    __syncthreads();
    float* tile = reinterpret_cast<float*>(smem) + wave * 32 * kStride;
    const bool gate = out.act == MXFP4_ACT_SWIGLU;
    const int columns = gate ? out.n >> 1 : out.n, piece = gate ? 16 : 8, pieces = kCols / piece, n1 = n0 + wn * kCols;
#pragma unroll
    for (int i = 0; i < MF; ++i) {
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<f32x4_t*>(tile + li * kStride + f * 32 + 16 * lh + e) =
                    f32x4_t{acc[i][f][e], acc[i][f][e + 1], acc[i][f][e + 2], acc[i][f][e + 3]};
        const int m1 = m0 + (wm * MF + i) * 32;
#pragma unroll 1
        for (int at = lane; at < 32 * pieces; at += 64) {
            const int row = at / pieces, n = at % pieces * piece;
            if (m1 + row >= out.m || n1 + n >= out.n)
                continue;
            float z[16];
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                if (e < 8 || gate) {
                    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(tile + row * kStride + n + e);
                    z[e] = v[0], z[e + 1] = v[1], z[e + 2] = v[2], z[e + 3] = v[3];
                }
            }
            if (out.bias)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if ((e < 8 || gate) && n1 + n + e < out.n)
                        z[e] += bf16_bits_to_f32(out.bias[n1 + n + e]);
            if (gate)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    z[e] = silu_gate(z[2 * e], z[2 * e + 1]);
            finish8(out, wide, m1 + row, (n1 + n) >> (gate ? 1 : 0), columns, z);
        }
    }
}

template <int WM, int WN, int MF, int NF>
hipError_t launch(const A8Args& a, hipStream_t stream)
{
    constexpr int BM = WM * MF * 32, BN = WN * NF * 32;
    static LdsLimit limit;
    const hipError_t raised = limit.raise(reinterpret_cast<const void*>(w4a8_block_kernel<WM, WN, MF, NF>), lds_bytes(BM, BN));
    if (raised != hipSuccess)
        return raised;
    auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
    const bool wide = aligned(a.y) && a.ldy % 8 == 0 && aligned(a.epi.residual) && (!a.epi.residual || a.ldr % 8 == 0);
    const int64_t tiles_n = (a.n + BN - 1) / BN, most = max(((int64_t)1 << 22) / tiles_n, (int64_t)1) * BM;
    for (int64_t at = 0; at < a.m; at += most) {
        const int m = (int)min(most, a.m - at), tiles_m = (m + BM - 1) / BM;
        const Out out = {a.epi.bias, a.epi.residual ? a.epi.residual + at * a.ldr : nullptr, a.y + at * a.ldy, a.ldy, a.ldr, m, a.n, a.epi.act};
        w4a8_block_kernel<WM, WN, MF, NF><<<dim3((unsigned)(tiles_m * tiles_n)), 512, lds_bytes(BM, BN), stream>>>(
            a.x + at * a.k, a.xs + at * (a.k >> 5), a.q, a.s, a.k, tiles_m, (int)tiles_n, wide, out);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_block(const A8Args& a, int shape, hipStream_t stream)
{
    switch (shape) {
    case 0:
        return launch<2, 4, 4, 2>(a, stream);
    case 1:
        return launch<2, 4, 2, 2>(a, stream);
    case 2:
        return launch<2, 4, 2, 1>(a, stream);
    default:
        return launch<2, 4, 1, 1>(a, stream);
    }
}

}  // namespace a8
}  // namespace mxfp4
