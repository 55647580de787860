// Low-rank adapters of many requests beside a shared projection:  y[m] = base[m] + scale[i] * B_i (A_i x[m]),  i = ids[m].
//
// The products give a workgroup rows of one adapter at a time, as the columns of v_mfma_f32_16x16x32_bf16: what another request's adapter holds
// (NaN, infinities) never meets a row, and rows may lie in any order.  Below 512 rows a workgroup has an adapter (grid z) and collects its rows from
// all of the call, so that an adapter's matrices are read once whatever the order (96 rows of 60 adapters at 4096 -> 12288, rank 32: 17 us, and 47
// with tiles of neighbouring rows); from 512 rows on, where reading all ids would cost more than it saves, it has 16 RT rows side by side and goes
// through the adapters among them.
//   shrink  t = A_i x for a part of K (grid y).  Rows of x and of A_i come into the LDS a phase of elements at a time by loads that write it directly,
//           D - 1 phases ahead, up to 512 bytes of a row side by side (in the layout of the matrix instruction a load touches a line per lane, and a
//           unit gets 38 bytes a ns instead of up to 150).  The waves that share a phase's elements add their sums in wave order; the parts' sums
//           lie in the workspace in FP32, side by side.
//   sum     adds the parts in order, scales t and cuts it into two BF16 numbers (together 16 bits, so that t's rounding does not show beside that
//           of y).  Below 512 rows the next step does it: a launch costs more than doing it several times.
//   expand  multiplies with B_i's rows, which are one piece of memory, and adds the base to the FP32 sums: one rounding.
// 5003 rows of five adapters, 8192 -> 8192, rank 64: shrink 30 us (x alone is 17 at a copy's rate), sum 5, expand 48 (base and y: 33).  The products
// by themselves are 25 us of the last, loads and stores 36: they overlap in part.  No gain: 16 or 64 rows a workgroup, two walks or eight, three
// phases ahead in one workgroup a unit, t's sums in every workgroup of expand (61 us), a whole line of a row an instruction.
#include "cast_block8.h"
#include "gemm_a8.h"

namespace mxfp4 {

namespace {

using a8::direct;
using a8::kOob;
using a8::lds_address;
using a8::past;
using a8::words;

__device__ __forceinline__ bf16x8_t load8(const void* p) { return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(p)); }

// Matrix instructions run with all lanes.  Where their result is used by some lanes only, the compiler may move them behind that
// condition, and the operands of the other lanes with it; this keeps them in front.
__device__ __forceinline__ void settle(f32x4_t& v) { asm volatile("" : "+v"(v)); }

__device__ __forceinline__ u32x4_t words16(const uint16_t* p, int64_t bytes)
{
    return words(reinterpret_cast<const uint8_t*>(p), (int)min(bytes, (int64_t)0x7FFFFF00));
}

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
    const int part = kFew ? (int)blockIdx.y : (int)(blockIdx.x % a.splits);
    extern __shared__ __align__(16) uint8_t all_lds[];
    uint16_t* list = reinterpret_cast<uint16_t*>(all_lds);
    uint8_t* smem = all_lds + (kFew ? kListBytes : 0);
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave % WK, wr = wave / WK;
    const int k0 = part * k_part, k1 = min(a.k, k0 + k_part), phases = (k1 - k0 + kPhase - 1) / kPhase;
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
                *reinterpret_cast<f32x4_t*>(a.part + ((int64_t)part * a.m + m0 + row) * a.r + rank) = sum;
        }
    };

    if constexpr (kFew) {
        int cur;
        const int count = collect(a, blockIdx.z, lane, list, cur);
        __syncthreads();
        for (int first = (int)blockIdx.x * (16 * RT); first < count; first += (int)gridDim.x * (16 * RT))
            tile(cur, 0, a.m, [&](int j) { return first + j < count ? (int)list[first + j] : -1; });
    } else {
        const int64_t m0 = (int64_t)(blockIdx.x / a.splits) * (16 * RT);
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

// Four ranks of t: their parts added in order, scaled, and cut into two BF16 numbers each: the four upper ones, the four lower ones.
__device__ __forceinline__ u32x4_t sum_of(const LoraArgs& a, int64_t at, float scale)
{
    f32x4_t v[kLoraSplits], t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < kLoraSplits; ++p)                       // (all loads at once; without conditions, which the compiler makes a way each of)
        v[p] = *reinterpret_cast<const f32x4_t*>(a.part + (int64_t)min(p, a.splits - 1) * a.m * a.r + at);
#pragma unroll
    for (int p = 0; p < kLoraSplits; ++p)
        t += p < a.splits ? v[p] : f32x4_t{0.f, 0.f, 0.f, 0.f};
    t *= scale;
    u32x4_t o;
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
        // cut off, not rounded: the largest numbers stay finite; an infinity leaves no rest
        auto cut = [](float v) { return v == v ? __float_as_uint(v) >> 16 : 0x7FC0u; };
        auto rest = [](float v) { const float d = v - __uint_as_float(__float_as_uint(v) & 0xFFFF0000u); return d == d ? d : 0.f; };
        o[e >> 1] = cut(t[e]) | cut(t[e + 1]) << 16;
        o[2 + (e >> 1)] = f32_to_bf16_rne2(rest(t[e]), rest(t[e + 1]));
    }
    return o;
}

// From 512 rows on: t of every row in place of its first part, eight upper numbers and eight lower ones of a thread's eight ranks, so that the
// workgroups that share a row's outputs read it once, and as the matrix instructions take it.
__global__ __launch_bounds__(256) void lora_sum_kernel(LoraArgs a)
{
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= (int64_t)a.m * a.r)
        return;
    const int id = a.ids[at / a.r];
    if (id < 0 || id >= a.adapters)
        return;
    const float scale = a.scales ? a.scales[id] : 1.f;
    const u32x4_t low = sum_of(a, at, scale), high = sum_of(a, at + 4, scale);
    *reinterpret_cast<u32x4_t*>(a.part + at) = u32x4_t{low[0], low[1], high[0], high[1]};
    *reinterpret_cast<u32x4_t*>(a.part + at + 4) = u32x4_t{low[2], low[3], high[2], high[3]};
}

// A wave has 64 outputs of the rows at a time; a workgroup's four lie side by side.  Row 16 f + i of the matrix instructions' B is output
// 32 (f / 2) + 8 (i / 4) + 4 (f % 2) + i % 4 of the 64: so a lane's four sums of two instructions are eight outputs side by side, 16 bytes of y,
// and four lanes have 64 bytes of a row.
constexpr int expand_stride(int kc) { return 8 * kc + 8; }                      // (16 bytes more: rows start in different banks)
constexpr int expand_t(int kc) { return 16 * expand_stride(kc) * 4; }

// KC chunks of eight ranks, 4, 8 or 16: a smaller rank is padded with zeros (loads past a row's end), so that places are shifts and no divisions.
// LDS: below 512 rows t's two halves [16][8 KC + 8]; for each wave B's rows [64][8 KC], chunk c of row r at c ^ (r / (16 / KC) % KC).
template <int KC>
struct Expand {
    const LoraArgs& a;
    uint8_t* smem;
    int lane, wave;
    static constexpr int kStride = expand_stride(KC), kTurn = 16 / KC;

    // B's rows n0 .. n0 + 63: one piece of memory, 1 KiB a load, each chunk to its place
    __device__ __forceinline__ void fetch(uint32_t to, int cur, int n0) const
    {
        const int cols = max(min(64, a.n - n0), 0);
        const u32x4_t rb = words16(a.b + ((int64_t)cur * a.n + n0) * a.r, (int64_t)cols * a.r * 2);
#pragma unroll
        for (int u = 0; u < KC; ++u) {
            const int slot = u * 64 + lane, row = slot / KC, f = row >> 4, i = row & 15, c = (slot % KC) ^ (row / kTurn % KC);
            const int out = 32 * (f >> 1) + 8 * (i >> 2) + 4 * (f & 1) + (i & 3);
            direct(to + u * 1024, c * 8 < a.r ? out * (a.r * 2) + c * 16 : kOob, rb, 0);
        }
    }

    // t of a tile's rows
    template <class RowOf>
    __device__ __forceinline__ void sums(float scale, RowOf row_of) const
    {
        uint16_t *hi = reinterpret_cast<uint16_t*>(smem), *lo = hi + 16 * kStride;
        for (int at = threadIdx.x; at < 16 * 2 * KC; at += 256) {
            const int j = at / (2 * KC), rank = at % (2 * KC) * 4, row = row_of(j);
            const u32x4_t t = row >= 0 && rank < a.r ? sum_of(a, (int64_t)row * a.r + rank, scale) : u32x4_t{0, 0, 0, 0};
            *reinterpret_cast<u32x2_t*>(hi + j * kStride + rank) = u32x2_t{t[0], t[1]};
            *reinterpret_cast<u32x2_t*>(lo + j * kStride + rank) = u32x2_t{t[2], t[3]};
        }
    }

    // This lane's outputs of the rows: 16 i + lane % 16, outputs n .. n + 7 and n + 32 .. n + 39, n = n0 + 8 (lane / 16).  Buffer instructions, which
    // leave out what lies past a descriptor's end: a condition would be a branch each, with a wait for its load at its end.
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const uint16_t* p, int64_t ld, int rows) const
    {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p), 0, p ? (int)(rows * ld * 2) : 0, 0x00020000);
    }

    __device__ __forceinline__ int offset(int row, int64_t ld) const { return row >= 0 ? row * (int)(ld * 2) : kOob; }

    template <int RT>
    __device__ __forceinline__ void load(u32x4_t (&v)[RT][2], __amdgpu_buffer_rsrc_t base, int n0, const int (&off)[RT]) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = n0 + 32 * h + 8 * (lane >> 4);
#pragma unroll
            for (int i = 0; i < RT; ++i)
                v[i][h] = __builtin_amdgcn_raw_buffer_load_b128(base, n < a.n ? (int)((uint32_t)off[i] + n * 2) : kOob, 0, 0);
        }
    }

    template <int RT>
    __device__ __forceinline__ void store(const u32x4_t (&v)[RT][2], __amdgpu_buffer_rsrc_t y, int n0, const int (&off)[RT]) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int n = n0 + 32 * h + 8 * (lane >> 4);
#pragma unroll
            for (int i = 0; i < RT; ++i)
                __builtin_amdgcn_raw_buffer_store_b128(v[i][h], y, n < a.n ? (int)((uint32_t)off[i] + n * 2) : kOob, 0, 0);
        }
    }

    // out = v + t B, B's rows at `b` in the LDS; t's numbers of row 16 i + lane % 16 and ranks 32 q + 8 (lane / 16) .. + 7: ranks_of(i, q, upper or lower)
    template <int RT, class RanksOf>
    __device__ __forceinline__ void product(u32x4_t (&out)[RT][2], const u32x4_t (&v)[RT][2], const uint8_t* b, RanksOf ranks_of) const
    {
        const int li = lane & 15, lg = lane >> 4;
        f32x4_t acc[RT][4] = {};
#pragma unroll
        for (int q = 0; q < KC / 4; ++q) {
            bf16x8_t w[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int row = 16 * f + li;
                w[f] = load8(b + (row * KC + ((4 * q + lg) ^ (row / kTurn % KC))) * 16);
            }
#pragma unroll
            for (int part = 1; part >= 0; --part)               // (the lower numbers first: small before large)
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const bf16x8_t t = ranks_of(i, q, part);
#pragma unroll
                    for (int f = 0; f < 4; ++f)
                        acc[i][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[f], t, acc[i][f], 0, 0, 0);
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
                    out[i][f >> 1][2 * (f & 1) + e] = f32_to_bf16_rne2(__uint_as_float(o << 16) + acc[i][f][2 * e], __uint_as_float(o & 0xFFFF0000u) + acc[i][f][2 * e + 1]);
                }
            }
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                asm volatile("" : "+v"(out[i][h]));             // (here, not behind the loads of the next v)
    }
};

// Below 512 rows: grid z an adapter, x 256 outputs of one of its tiles of 16 rows (and every gridDim.y-th), y the tile.  B's rows stay for all tiles.
template <int KC>
__global__ __launch_bounds__(256, 4) void lora_expand_few_kernel(LoraArgs a)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Expand<KC> e{a, smem + kListBytes, (int)threadIdx.x & 63, wave};
    uint16_t* list = reinterpret_cast<uint16_t*>(smem);
    int cur;
    const int count = collect(a, (int)blockIdx.z + 1 < (int)gridDim.z ? (int)blockIdx.z : -1, e.lane, list, cur);
    const int n0 = ((int)blockIdx.x * 4 + wave) * 64;
    int first = (int)blockIdx.y * 16;
    if (first >= count || (cur < 0 && a.base == a.y))
        return;
    const int own = expand_t(KC) + wave * (1024 * KC);
    if (cur >= 0)
        e.fetch(lds_address(e.smem) + own, cur, n0);
    const float scale = a.scales && cur >= 0 ? a.scales[cur] : 1.f;
    const auto base = e.rows_of(a.base, a.ldb, a.m), y = e.rows_of(a.y, a.ldy, a.m);
    __syncthreads();
    for (bool next = false; first < count; first += (int)gridDim.y * 16, next = true) {
        auto row_of = [&](int j) { return first + j < count ? (int)list[first + j] : -1; };
        const int row = row_of(e.lane & 15), from[1] = {e.offset(row, a.ldb)}, to[1] = {e.offset(row, a.ldy)};
        u32x4_t v[1][2], out[1][2];
        e.load(v, base, n0, from);
        if (cur >= 0) {
            if (next)
                __syncthreads();                                // (t has been read)
            e.sums(scale, row_of);
            drain_vmem();
            __syncthreads();
            e.product(out, v, e.smem + own, [&](int, int q, int part) {
                return load8(reinterpret_cast<const uint16_t*>(e.smem) + (16 * part + (e.lane & 15)) * e.kStride + 32 * q + 8 * (e.lane >> 4));
            });
        }
        e.store(cur >= 0 ? out : v, y, n0, to);
    }
}

// Grid x: `walks` times 256 outputs, those of 16 RT rows side by side, then the next rows' (a piece of B stays with a die); the adapters among the rows are
// shared out over grid z.
template <int KC, int RT>
__global__ __launch_bounds__(256, KC == 16 ? 2 : 3) void lora_expand_kernel(LoraArgs a, int walks, int chunks)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Expand<KC> e{a, smem, (int)threadIdx.x & 63, wave};
    const int64_t m0 = (int64_t)(blockIdx.x / chunks) * (16 * RT);
    const int rows = (int)min((int64_t)16 * RT, a.m - m0);
    const int id = tile_ids(a, m0, rows, e.lane);
    const int own = wave * (1024 * KC);
    const uint64_t some = __ballot(id >= 0);
    const uint64_t none = blockIdx.z == 0 && a.base != a.y ? __ballot(id < 0 && e.lane < rows) : 0;    // rows of no adapter: the base as it is
    const auto output = [&](int walk) { return (((int)(blockIdx.x % chunks) * walks + walk) * 4 + wave) * 64; };
    const auto base = e.rows_of(a.base ? a.base + m0 * a.ldb : nullptr, a.ldb, rows), y = e.rows_of(a.y + m0 * a.ldy, a.ldy, rows);
    u32x4_t v[RT][2], out[RT][2];
    int from[RT], to[RT];
    const auto take = [&](uint64_t mine) {
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int row = mine >> (16 * i + (e.lane & 15)) & 1 ? 16 * i + (e.lane & 15) : -1;
            from[i] = e.offset(row, a.ldb);
            to[i] = e.offset(row, a.ldy);
        }
    };
    take(none);
    for (int walk = 0; none && walk < walks; ++walk) {
        e.load(v, base, output(walk), from);
        e.store(v, y, output(walk), to);
    }
    if (!some)
        return;
    // t of all rows: what a row is of another adapter than the one whose B is multiplied meets no row of that one.
    const auto sums = __builtin_amdgcn_make_buffer_rsrc(a.part + m0 * a.r, 0, rows * a.r * 4, 0x00020000);
    bf16x8_t t[RT][KC / 4][2];
    uint64_t todo = some;
    bool first = true;
    for (int nth = 0; todo; ++nth) {
        const int cur = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
        const uint64_t mine = __ballot(id == cur);
        todo &= ~mine;
        if (nth % (int)gridDim.z != (int)blockIdx.z)
            continue;
        take(mine);
        e.fetch(lds_address(smem) + own, cur, output(0));
        e.load(v, base, output(0), from);
        if (first) {
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int q = 0; q < KC / 4; ++q)
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        const int row = 16 * i + (e.lane & 15), rank = 32 * q + 8 * (e.lane >> 4);
                        t[i][q][part] = __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(sums, rank < a.r ? (row * a.r + rank + 4 * part) * 4 : kOob, 0, 0));
                    }
            first = false;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        // The next outputs' rows of B and base are on their way before this walk's outputs leave, and the wait for them does not wait for the stores.
        for (int walk = 0; walk < walks; ++walk) {
            e.product(out, v, smem + own, [&](int i, int q, int part) { return t[i][q][part]; });
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the wave's part has been read)
            if (walk + 1 < walks) {
                e.fetch(lds_address(smem) + own, cur, output(walk + 1));
                e.load(v, base, output(walk + 1), from);
            }
            e.store(out, y, output(walk), to);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * RT) : "memory");
        }
    }
}


// Workgroups of a grid are limited, and so is the reach of an offset into x, base and y: very many rows, and rows very far apart, are several pairs of launches.
template <int RT, int RG, int WK, int D, bool kFew>
hipError_t launch(LoraArgs a, hipStream_t stream)
{
    constexpr int KC = RG <= 2 ? 4 : RG <= 4 ? 8 : 16, ET = kFew ? 1 : 2;
    static LdsLimit shrink, expand;
    const int list = kFew ? kListBytes : 0, shrink_bytes = shrink_lds(RT, RG, WK, D) + list, expand_bytes = 4 * 1024 * KC + (kFew ? list + expand_t(KC) : 0);
    const void* second;
    if constexpr (kFew)
        second = reinterpret_cast<const void*>(lora_expand_few_kernel<KC>);
    else
        second = reinterpret_cast<const void*>(lora_expand_kernel<KC, ET>);
    hipError_t e = shrink.raise(reinterpret_cast<const void*>(lora_shrink_kernel<RT, RG, WK, D, kFew>), shrink_bytes);
    if (e == hipSuccess)
        e = expand.raise(second, expand_bytes);
    const int k_part = ((a.k + a.splits - 1) / a.splits + phase_of(WK) - 1) / phase_of(WK) * phase_of(WK);
    const int64_t pieces = ((int64_t)a.m + 16 * ET - 1) / (16 * ET) * (((int64_t)a.n + 255) / 256);
    const int walks = kFew ? 1 : (int)min(max(pieces / 768, (int64_t)1), (int64_t)4), step = 256 * walks, chunks = (int)(((int64_t)a.n + step - 1) / step);
    const int64_t all = a.m, most = kFew ? min(all, ((int64_t)1 << 29) / max(a.ldx, max(a.ldb, a.ldy))) : max((1 << 20) / chunks, 1) * (16 * RT * ET);
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
            lora_expand_few_kernel<KC><<<dim3(chunks, share, groups + 1), 256, expand_bytes, stream>>>(b);
        } else {
            const int wide = (b.m + ET * 16 - 1) / (ET * 16);
            // (tiles with rows of several adapters: two workgroups share them in shrink, 24 us for 27; in expand one goes through them, 48 for 52)
            const auto slots = [&](int64_t least, int64_t others) { return (int)min((int64_t)min(a.adapters, 16), max(1024 / others, least)); };
            lora_shrink_kernel<RT, RG, WK, D, false><<<dim3(tiles * a.splits, 1, slots(2, (int64_t)tiles * a.splits)), 512, shrink_bytes, stream>>>(b, k_part);
            lora_sum_kernel<<<(unsigned)(((int64_t)b.m * (a.r / 8) + 255) / 256), 256, 0, stream>>>(b);
            lora_expand_kernel<KC, ET><<<dim3(wide * chunks, 1, slots(1, (int64_t)wide * chunks)), 256, expand_bytes, stream>>>(b, walks, chunks);
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
    if (few(m))
        return (int)(most < kLoraSplits ? most : kLoraSplits);
    // a power of two: neighbouring workgroups have the parts in turn, so a part of A's columns stays with the dies that have it
    int s = kLoraSplits;
    while (s > 1 && (s > most || s * tiles > 1024))
        s /= 2;
    return s;
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
           : groups <= 4 ? launch<4, 4, 2, 3, false>(a, stream)
                         : launch<2, 8, 4, 2, false>(a, stream);
}

}  // namespace mxfp4
