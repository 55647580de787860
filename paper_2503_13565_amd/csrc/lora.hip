// Low-rank adapters of many requests beside a shared projection:  y[m] = base[m] + scale[i] * B_i (A_i x[m]),  i = ids[m].
//
// Two launches.  Both give a workgroup rows of one adapter at a time, as the columns of v_mfma_f32_16x16x32_bf16: what another request's adapter
// holds (NaN, infinities) never meets a row, and rows may lie in any order.  Below 512 rows a workgroup has an adapter (grid z) and collects
// its rows from all of the call, so that an adapter's matrices are read once whatever the order; from 512 rows on, where reading all ids would
// cost more than it saves, it has 16 RT rows side by side and goes through the adapters among them.
//   shrink  t = A_i x for a part of K (grid y).  Rows of x and of A_i come into the LDS a phase of elements at a time by loads that write it directly,
//           D - 1 phases ahead, up to 512 bytes of a row side by side (in the layout of the matrix instruction a load touches a line per lane, and a
//           unit gets 38 bytes a ns instead of up to 150).  The waves that share a phase's elements add their sums in wave order; the parts' sums
//           lie in the workspace in FP32, side by side.
//   expand  adds the parts in order, scales t and cuts it into two BF16 numbers (together 16 bits, so that t's rounding does not show beside that of
//           y), multiplies with B_i's rows, which are one piece of memory, and adds the base to the FP32 sums: one rounding.
#include "cast_block8.h"
#include "gemm_a8.h"

namespace mxfp4 {

namespace {

using a8::direct;
using a8::kOob;
using a8::lds_address;
using a8::past;
using a8::turn;
using a8::words;

__device__ __forceinline__ bf16x8_t load8(const void* p) { return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(p)); }

// Matrix instructions run with all lanes.  Where their result is used by some lanes only, the compiler may move them behind that
// condition, and the operands of the other lanes with it; this keeps them in front.
__device__ __forceinline__ void settle(f32x4_t& v) { asm volatile("" : "+v"(v)); }

__device__ __forceinline__ u32x4_t words16(const uint16_t* p, int64_t bytes)
{
    return words(reinterpret_cast<const uint8_t*>(p), (int)min(bytes, (int64_t)0x7FFFFF00));
}

constexpr int kRanks = 128;             // the largest rank of a call
constexpr int kLoraSplits = 8;          // parts of K

// The adapter of each of the tile's 16 RT rows, in the lane of its number; -1: none.
__device__ __forceinline__ int tile_ids(const LoraArgs& a, int64_t m0, int rows, int lane)
{
    const int id = lane < rows ? a.ids[m0 + lane] : -1;
    return id >= 0 && id < a.adapters ? id : -1;
}

// Below 512 rows: grid z is an adapter, or where there are more adapters than rows, the row that is its adapter's first.  The adapter's rows, in order,
// go into `list` (every wave writes the same), their number comes back; z of gridDim.z - 1 has the rows of no adapter.
constexpr int kFewRows = 512, kListBytes = kFewRows * 2;
__device__ __forceinline__ int collect(const LoraArgs& a, int z, int lane, uint16_t* list, int& cur)
{
    int id[kFewRows / 64];
#pragma unroll
    for (int u = 0; u < kFewRows / 64; ++u) {
        const int row = u * 64 + lane, v = row < a.m ? a.ids[row] : -2;
        id[u] = v == -2 && row >= a.m ? -2 : v >= 0 && v < a.adapters ? v : -1;
    }
    const bool by_row = a.adapters > a.m;
    cur = z;
    if (z < 0)
        cur = -1;
    else if (by_row)
        cur = a.ids[z];
    if (z >= 0 && (cur < 0 || cur >= a.adapters))
        return 0;
    int count = 0;
#pragma unroll
    for (int u = 0; u < kFewRows / 64; ++u) {
        if (u * 64 >= a.m)
            break;
        const uint64_t mine = __ballot(id[u] == cur);
        if (by_row && z >= 0 && count == 0 && mine && u * 64 + __builtin_ctzll(mine) != z)
            return 0;
        if (id[u] == cur)
            list[count + __builtin_popcountll(mine & ((1ull << lane) - 1))] = (uint16_t)(u * 64 + lane);
        count += __builtin_popcountll(mine);
    }
    return count;
}

// The eight waves are 8 / WK x WK: WK share a phase's elements, 32 each, the others the tile's rows.
constexpr int phase_of(int wk) { return 32 * wk; }
constexpr int shrink_buffer(int rt, int rg, int wk) { return (rt + rg) * 16 * 64 * wk; }
constexpr int shrink_lds(int rt, int rg, int wk, int d)
{
    const int buffers = d * shrink_buffer(rt, rg, wk), sums = wk * rt * rg * 1024;
    return buffers > sums ? buffers : sums;
}

template <int RT, int RG, int WK, int D, bool kFew>
__global__ __launch_bounds__(512) void lora_shrink_kernel(LoraArgs a, int k_part)
{
    constexpr int kPhase = phase_of(WK), kBuf = shrink_buffer(RT, RG, WK), kRow = 64 * WK, kChunks = kRow / 16;
    constexpr int WR = 8 / WK, MR = RT / WR, C = (RT + RG) * WK / 8, kX = RT * WK;           // loads of a wave, KiB of x
    static_assert(MR * WR == RT && C * 8 == (RT + RG) * WK && kX % 8 == 0, "whole tiles and loads a wave");
    extern __shared__ __align__(16) uint8_t all_lds[];
    uint16_t* list = reinterpret_cast<uint16_t*>(all_lds);
    uint8_t* smem = all_lds + (kFew ? kListBytes : 0);
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave % WK, wr = wave / WK;
    const int k0 = (int)blockIdx.y * k_part, k1 = min(a.k, k0 + k_part), phases = (k1 - k0 + kPhase - 1) / kPhase;
    const uint32_t lds_at = lds_address(smem);
    bool used = false;

    // Row j of the tile's is row_of(j) of x, behind row m0; below 0: none.
    auto tile = [&](int cur, int64_t m0, int reach, auto row_of) {
        const u32x4_t rx = words16(a.x + m0 * a.ldx, (int64_t)reach * a.ldx * 2), ra = words16(a.a + (int64_t)cur * a.r * a.k, (int64_t)a.r * a.k * 2);
        // Load c of wave w fills KiB 8 c + w of a phase: x first, A behind it.  Chunk c of row r lies at c ^ (r % 16).
        int off[C], chunk[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int piece = (c * 8 + wave) * 64 + lane, line = piece / kChunks;
            const int row = c * 8 < kX ? row_of(line) : line - RT * 16;
            chunk[c] = (piece % kChunks) ^ (line & 15 & (kChunks - 1));
            const bool live = c * 8 < kX ? row >= 0 : row < a.r;
            off[c] = live ? (int)(row * (c * 8 < kX ? a.ldx : (int64_t)a.k) + k0) * 2 + chunk[c] * 16 : kOob;
        }
        auto issue = [&](int p, int b) {                        // (past the part's end: zeros, so that the loads of a phase are as many)
            const int from = p < phases ? p * (kPhase * 2) : 0;
#pragma unroll
            for (int c = 0; c < C; ++c)
                direct(lds_at + b * kBuf + (c * 8 + wave) * 1024, off[c] | past((k1 - k0) / 8 - 1, p * (kPhase / 8) + chunk[c]), c * 8 < kX ? rx : ra, from);
        };
        if (used)
            __syncthreads();                                    // (the sums of the tile before have been read)
        used = true;
#pragma unroll
        for (int d = 0; d < D; ++d)
            issue(d, d);
        f32x4_t acc[MR][RG] = {};
        int b = 0;
        for (int p = 0; p < phases; ++p) {
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * C) : "memory");
            lds_barrier();
            const uint8_t* at = smem + b * kBuf + li * kRow + ((4 * wk + lg) ^ (li & (kChunks - 1))) * 16;
            bf16x8_t x[MR], w[RG];
#pragma unroll
            for (int f = 0; f < MR; ++f)
                x[f] = load8(at + (wr * MR + f) * (16 * kRow));
#pragma unroll
            for (int f = 0; f < RG; ++f)
                w[f] = load8(at + (RT + f) * (16 * kRow));
            lds_barrier();                                      // every wave has read the buffer
            issue(p + D, b);
#pragma unroll
            for (int i = 0; i < MR; ++i)
#pragma unroll
                for (int f = 0; f < RG; ++f)
                    acc[i][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[f], x[i], acc[i][f], 0, 0, 0);
            b = b == D - 1 ? 0 : b + 1;
        }
        drain_vmem();                                           // (the loads behind the last phase write the LDS)
        __syncthreads();
        f32x4_t* red = reinterpret_cast<f32x4_t*>(smem);
#pragma unroll
        for (int i = 0; i < MR; ++i)
#pragma unroll
            for (int f = 0; f < RG; ++f)
                red[(wk * (RT * RG) + (wr * MR + i) * RG + f) * 64 + lane] = acc[i][f];
        __syncthreads();
        for (int at = threadIdx.x; at < RT * RG * 64; at += 512) {
            const int f = at >> 6, l = at & 63, row = row_of(f / RG * 16 + (l & 15)), rank = f % RG * 16 + 4 * (l >> 4);
            f32x4_t sum = red[at];
#pragma unroll
            for (int w = 1; w < WK; ++w)
                sum += red[w * (RT * RG * 64) + at];
            if (row >= 0 && rank < a.r)
                *reinterpret_cast<f32x4_t*>(a.part + ((int64_t)blockIdx.y * a.m + m0 + row) * a.r + rank) = sum;
        }
    };

    if constexpr (kFew) {
        int cur;
        const int count = collect(a, blockIdx.z, lane, list, cur);
        __syncthreads();
        for (int first = (int)blockIdx.x * (16 * RT); first < count; first += (int)gridDim.x * (16 * RT))
            tile(cur, 0, a.m, [&](int j) { return first + j < count ? (int)list[first + j] : -1; });
    } else {
        const int64_t m0 = (int64_t)blockIdx.x * (16 * RT);
        const int rows = (int)min((int64_t)16 * RT, a.m - m0), id = tile_ids(a, m0, rows, lane);
        uint64_t todo = __ballot(id >= 0);
        for (int nth = 0; todo; ++nth) {
            const int cur = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
            const uint64_t mine = __ballot(id == cur);
            todo &= ~mine;
            if (nth % (int)gridDim.z == (int)blockIdx.z)
                tile(cur, m0, rows, [&](int j) { return mine >> j & 1 ? j : -1; });
        }
    }
}

// A wave has 64 outputs of the rows at a time; a workgroup's four lie side by side.  Row 16 f + i of the matrix instructions' B is output
// 32 (f / 2) + 8 (i / 4) + 4 (f % 2) + i % 4 of the 64: so a lane's four sums of two instructions are eight outputs side by side, 16 bytes of y,
// and four lanes have 64 bytes of a row.
constexpr int expand_stride(int r) { return ((r + 31) & ~31) + 8; }             // (16 bytes more: rows start in different banks)
constexpr int expand_t(int rt, int r) { return rt * 16 * expand_stride(r) * 4; }
constexpr int expand_lds(int rt, int r) { return expand_t(rt, r) + 4 * 128 * r; }

// LDS: t's two halves [16 RT][ranks + 8], and for each wave B's rows [64][r], chunks turned where their number is a power of two
struct Expand {
    const LoraArgs& a;
    uint8_t* smem;
    int lane, wave;

    __device__ __forceinline__ int place(int row, int c) const
    {
        const int chunks = a.r >> 3;
        if (chunks & (chunks - 1))
            return c;
        return c ^ (chunks >= 16 ? row & 15 : row / (16 / chunks) & (chunks - 1));
    }

    // B's rows n0 .. n0 + 63: one piece of memory, 1 KiB a load, each chunk to its place
    __device__ __forceinline__ void fetch(uint32_t to, int cur, int n0) const
    {
        const int chunks = a.r >> 3, cols = max(min(64, a.n - n0), 0);
        const u32x4_t rb = words16(a.b + ((int64_t)cur * a.n + n0) * a.r, (int64_t)cols * a.r * 2);
        for (int u = 0; u < chunks; ++u) {
            const int slot = u * 64 + lane, row = slot / chunks, f = row >> 4, i = row & 15;
            const int out = 32 * (f >> 1) + 8 * (i >> 2) + 4 * (f & 1) + (i & 3);
            direct(to + u * 1024, (out * chunks + place(row, slot - row * chunks)) * 16, rb, 0);
        }
    }

    template <int RT, class RowOf>
    __device__ __forceinline__ void sums(float scale, int64_t m0, RowOf row_of) const
    {
        const int quads = ((a.r + 31) & ~31) / 4, stride = expand_stride(a.r);
        uint16_t *hi = reinterpret_cast<uint16_t*>(smem), *lo = hi + RT * 16 * stride;
        for (int at = threadIdx.x; at < RT * 16 * quads; at += 256) {
            const int j = at / quads, rank = (at - j * quads) * 4, row = row_of(j);
            f32x4_t t = {0.f, 0.f, 0.f, 0.f};
            if (row >= 0 && rank < a.r) {
                const float* from = a.part + (m0 + row) * a.r + rank;
                f32x4_t v[kLoraSplits];
#pragma unroll
                for (int p = 0; p < kLoraSplits; ++p)
                    if (p < a.splits)
                        v[p] = *reinterpret_cast<const f32x4_t*>(from + (int64_t)p * a.m * a.r);
#pragma unroll
                for (int p = 0; p < kLoraSplits; ++p)
                    if (p < a.splits)
                        t += v[p];
                t *= scale;
            }
            u32x2_t h, l;
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                // cut off, not rounded: the largest numbers stay finite; an infinity leaves no rest
                auto cut = [](float v) { return v == v ? __float_as_uint(v) >> 16 : 0x7FC0u; };
                auto rest = [](float v) { const float d = v - __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); return d == d ? d : 0.f; };
                h[e >> 1] = cut(t[e]) | cut(t[e + 1]) << 16;
                l[e >> 1] = f32_to_bf16_rne2(rest(t[e]), rest(t[e + 1]));
            }
            *reinterpret_cast<u32x2_t*>(hi + j * stride + rank) = h;
            *reinterpret_cast<u32x2_t*>(lo + j * stride + rank) = l;
        }
    }

    // This lane's outputs of the rows: 16 i + lane % 16, outputs n .. n + 7 and n + 32 .. n + 39, n = n0 + 8 (lane / 16)
    template <int RT, class RowOf>
    __device__ __forceinline__ void load(u32x4_t (&base)[RT][2], int64_t m0, int n0, RowOf row_of) const
    {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int row = row_of(16 * i + (lane & 15)), n = n0 + 8 * (lane >> 4);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                base[i][h] = u32x4_t{0, 0, 0, 0};
                if (a.base && row >= 0 && n + 32 * h < a.n)
                    base[i][h] = *reinterpret_cast<const u32x4_t*>(a.base + (m0 + row) * a.ldb + n + 32 * h);
            }
        }
    }

    template <int RT, class RowOf>
    __device__ __forceinline__ void store(const u32x4_t (&v)[RT][2], int64_t m0, int n0, RowOf row_of) const
    {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int row = row_of(16 * i + (lane & 15)), n = n0 + 8 * (lane >> 4);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (row >= 0 && n + 32 * h < a.n)
                    *reinterpret_cast<u32x4_t*>(a.y + (m0 + row) * a.ldy + n + 32 * h) = v[i][h];
        }
    }

    // v + t B, B's rows at `b` in the LDS
    template <int RT>
    __device__ __forceinline__ void product(u32x4_t (&v)[RT][2], const uint8_t* b) const
    {
        const int li = lane & 15, lg = lane >> 4, chunks = a.r >> 3, stride = expand_stride(a.r);
        const uint16_t *hi = reinterpret_cast<const uint16_t*>(smem), *lo = hi + RT * 16 * stride;
        f32x4_t acc[RT][4] = {};
        for (int kk = 0; kk < a.r; kk += 32) {
            bf16x8_t w[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int row = 16 * f + li, c = (kk >> 3) + lg;
                w[f] = load8(b + (row * chunks + place(row, min(c, chunks - 1))) * 16);     // (past the rank, t is zero; infinities are not multiplied with it)
                if (c >= chunks)
                    w[f] = bf16x8_t{};
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const bf16x8_t th = load8(hi + (i * 16 + li) * stride + kk + 8 * lg), tl = load8(lo + (i * 16 + li) * stride + kk + 8 * lg);
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    acc[i][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[f], tl, acc[i][f], 0, 0, 0);
                    acc[i][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[f], th, acc[i][f], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                settle(acc[i][f]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t o = v[i][f >> 1][2 * (f & 1) + e];
                    v[i][f >> 1][2 * (f & 1) + e] = f32_to_bf16_rne2(__uint_as_float(o << 16) + acc[i][f][2 * e], __uint_as_float(o & 0xFFFF0000u) + acc[i][f][2 * e + 1]);
                }
            }
    }
};

// Below 512 rows: grid z an adapter, x 256 outputs of one of its tiles of 16 rows (and every gridDim.y-th), y the tile.  B's rows stay for all tiles.
__global__ __launch_bounds__(256, 4) void lora_expand_few_kernel(LoraArgs a)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Expand e{a, smem + kListBytes, (int)threadIdx.x & 63, wave};
    uint16_t* list = reinterpret_cast<uint16_t*>(smem);
    int cur;
    const int count = collect(a, (int)blockIdx.z + 1 < (int)gridDim.z ? (int)blockIdx.z : -1, e.lane, list, cur);
    const int n0 = ((int)blockIdx.x * 4 + wave) * 64;
    int first = (int)blockIdx.y * 16;
    if (first >= count || (cur < 0 && a.base == a.y))
        return;
    const int own = expand_t(1, a.r) + wave * (128 * a.r);
    if (cur >= 0)
        e.fetch(lds_address(e.smem) + own, cur, n0);
    const float scale = a.scales && cur >= 0 ? a.scales[cur] : 1.f;
    __syncthreads();
    for (bool next = false; first < count; first += (int)gridDim.y * 16, next = true) {
        auto row_of = [&](int j) { return first + j < count ? (int)list[first + j] : -1; };
        u32x4_t v[1][2];
        e.load<1>(v, 0, n0, row_of);
        if (cur >= 0) {
            if (next)
                __syncthreads();                                // (t has been read)
            e.sums<1>(scale, 0, row_of);
            drain_vmem();
            __syncthreads();
            e.product<1>(v, e.smem + own);
        }
        e.store<1>(v, 0, n0, row_of);
    }
}

// Grid x: `walks` times 256 outputs, those of 16 RT rows side by side, then the next rows' (a piece of B stays with a die); the adapters among the rows are
// shared out over grid z.
template <int RT>
__global__ __launch_bounds__(256, RT == 4 ? 2 : 4) void lora_expand_kernel(LoraArgs a, int walks, int chunks)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Expand e{a, smem, (int)threadIdx.x & 63, wave};
    const int64_t m0 = (int64_t)(blockIdx.x / chunks) * (16 * RT);
    const int rows = (int)min((int64_t)16 * RT, a.m - m0);
    const int id = tile_ids(a, m0, rows, e.lane);
    const int own = expand_t(RT, a.r) + wave * (128 * a.r);
    const uint64_t some = __ballot(id >= 0);
    const uint64_t none = blockIdx.z == 0 && a.base != a.y ? __ballot(id < 0 && e.lane < rows) : 0;    // rows of no adapter: the base as it is
    bool used = false;                                          // whether the LDS has been written
    int has = -1;                                               // whose t it holds
    for (int walk = 0; walk < walks; ++walk) {
        const int n0 = (((int)(blockIdx.x % chunks) * walks + walk) * 4 + wave) * 64;
        u32x4_t v[RT][2];
        if (none) {
            auto row_of = [&](int j) { return none >> j & 1 ? j : -1; };
            e.load<RT>(v, m0, n0, row_of);
            e.store<RT>(v, m0, n0, row_of);
        }
        uint64_t todo = some;
        for (int nth = 0; todo; ++nth) {
            const int cur = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
            const uint64_t mine = __ballot(id == cur);
            todo &= ~mine;
            if (nth % (int)gridDim.z != (int)blockIdx.z)
                continue;
            auto row_of = [&](int j) { return mine >> j & 1 ? j : -1; };
            e.load<RT>(v, m0, n0, row_of);
            if (used)
                __syncthreads();                                // (it has been read)
            used = true;
            e.fetch(lds_address(smem) + own, cur, n0);
            if (has != cur)                                     // (one adapter all walks long: t is there)
                e.sums<RT>(a.scales ? a.scales[cur] : 1.f, m0, row_of);
            has = cur;
            drain_vmem();
            __syncthreads();
            e.product<RT>(v, smem + own);
            e.store<RT>(v, m0, n0, row_of);
        }
    }
}

#ifndef LORA_ET
#define LORA_ET 2
#endif
constexpr int kExpandTiles = LORA_ET;

// Workgroups of a grid are limited, and so is the reach of an offset into x: very many rows, and rows very far apart, are several pairs of launches.
template <int RT, int RG, int WK, int D, bool kFew>
hipError_t launch(LoraArgs a, hipStream_t stream)
{
    constexpr int ET = kFew ? 1 : kExpandTiles;
    static LdsLimit shrink, expand;
    const int list = kFew ? kListBytes : 0, shrink_bytes = shrink_lds(RT, RG, WK, D) + list, expand_bytes = expand_lds(ET, a.r) + list;
    const void* second;
    if constexpr (kFew)
        second = reinterpret_cast<const void*>(lora_expand_few_kernel);
    else
        second = reinterpret_cast<const void*>(lora_expand_kernel<ET>);
    hipError_t e = shrink.raise(reinterpret_cast<const void*>(lora_shrink_kernel<RT, RG, WK, D, kFew>), shrink_bytes);
    if (e == hipSuccess)
        e = expand.raise(second, expand_lds(ET, kRanks) + list);
    const int k_part = ((a.k + a.splits - 1) / a.splits + phase_of(WK) - 1) / phase_of(WK) * phase_of(WK);
    const int walks = !kFew && a.n >= 2048 ? 4 : 1, step = 256 * walks, chunks = (int)(((int64_t)a.n + step - 1) / step);
    const int64_t all = a.m, most = kFew ? min(all, ((int64_t)1 << 29) / a.ldx) : max((1 << 21) / chunks, 1) * (16 * RT * ET);
    for (int64_t at = 0; at < all && e == hipSuccess; at += most) {
        LoraArgs b = a;
        b.m = (int)min(all - at, most);
        b.x += at * a.ldx;
        b.ids += at;
        b.base = a.base ? a.base + at * a.ldb : nullptr;
        b.y += at * a.ldy;
        const int tiles = (b.m + RT * 16 - 1) / (RT * 16);
        if constexpr (kFew) {
            const int groups = min(a.adapters, b.m), share = min(tiles, (2 * tiles + groups - 1) / groups);
            lora_shrink_kernel<RT, RG, WK, D, true><<<dim3(share, a.splits, groups), 512, shrink_bytes, stream>>>(b, k_part);
            lora_expand_few_kernel<<<dim3(chunks, share, groups + 1), 256, expand_bytes, stream>>>(b);
        } else {
            const int slots = min(a.adapters, 2), wide = (b.m + ET * 16 - 1) / (ET * 16);
            lora_shrink_kernel<RT, RG, WK, D, false><<<dim3(tiles, a.splits, slots), 512, shrink_bytes, stream>>>(b, k_part);
            lora_expand_kernel<ET><<<dim3(wide * chunks, 1, slots), 256, expand_bytes, stream>>>(b, walks, chunks);
        }
        e = hipGetLastError();
    }
    return e;
}

constexpr bool few(int64_t m) { return m < kFewRows; }

}  // namespace

int lora_splits(int64_t m, int64_t k, int64_t r)
{
    const int64_t rows = r > 64 ? 32 : 64, tiles = (m + rows - 1) / rows, phase = phase_of(few(m) ? 8 : 4), most = (k + phase - 1) / phase;
    int64_t s = few(m) ? kLoraSplits : 512 / tiles;
    s = s > kLoraSplits ? kLoraSplits : s;
    s = s > most ? most : s;
    return (int)(s < 1 ? 1 : s);
}

hipError_t launch_lora(const LoraArgs& a, const DeviceInfo&, hipStream_t stream)
{
    const int groups = (a.r + 15) / 16;
    if (few(a.m))
        return groups <= 1   ? launch<1, 1, 8, 4, true>(a, stream)
               : groups <= 2 ? launch<1, 2, 8, 3, true>(a, stream)
               : groups <= 4 ? launch<1, 4, 8, 2, true>(a, stream)
                             : launch<1, 8, 8, 2, true>(a, stream);
    return groups <= 2   ? launch<4, 2, 4, 2, false>(a, stream)
           : groups <= 4 ? launch<4, 4, 4, 2, false>(a, stream)
                         : launch<2, 8, 4, 2, false>(a, stream);
}

}  // namespace mxfp4
