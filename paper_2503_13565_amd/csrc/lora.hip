// Low-rank adapters of many requests beside a shared projection:  y[m] = base[m] + scale[i] * B_i (A_i x[m]),  i = ids[m].
//
// A workgroup of the products has rows of one adapter, as the columns of v_mfma_f32_16x16x32_bf16: what another request's adapter holds (NaN,
// infinities) never meets a row, rows may lie in any order, and an adapter's matrices are read once for all its rows (up to a workgroup's).
//   group   sorts the rows by adapter, in one workgroup: counts, sums over the adapters, places.  Rows of an adapter come in any order, which no output
//           depends on.  It costs 3 us for hundreds of rows and 7 for 5003, so up to 128 rows the products find theirs themselves (96 rows of 60
//           adapters at 4096 -> 12288, rank 32: 18 us for 20.4); with more of them, the sixteens of an adapter that has most of the rows would come one
//           after the other (256 rows of one among 60, 4096 -> 4096, rank 16: 12.3 us for 45), and tiles of neighbouring rows would read many
//           adapters' matrices each (512 rows of 60, 4096 -> 12288, rank 64: 47 us for 118).
//   shrink  t = A_i x for a part of K.  Rows of x and of A_i come into the LDS a phase of elements at a time by loads that write it directly,
//           D - 1 phases ahead, up to 512 bytes of a row side by side (in the layout of the matrix instruction a load touches a line per lane, and a
//           unit gets 38 bytes a ns instead of up to 150).  The waves that share a phase's elements add their sums in wave order; the parts' sums
//           lie in the workspace in FP32, side by side.
//   sum     adds the parts in order, scales t and cuts it into two BF16 numbers (together 16 bits, so that t's rounding does not show beside that
//           of y).  Below 512 rows the next step does it: a launch costs more than doing it several times.
//   expand  multiplies with B_i's rows, which are one piece of memory, and adds the base to the FP32 sums: one rounding.
// 5003 rows of five adapters, 8192 -> 8192, rank 64: group 7 us, shrink 24 (x alone is 17 at a copy's rate), sum 5, expand 46 (base and y: 33; the
// products by themselves are 25, loads and stores 36: they overlap in part).  No gain in expand: 16 or 64 rows a workgroup, two walks or eight, t's
// sums in every workgroup (61 us), a whole line of a row an instruction.  In one token's call (8 us) each launch is a chain of three loads;
// both products in one launch, with t made again by every workgroup, were as long at 4096 and longer beyond.
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
constexpr int kAlone = 128;             // the most rows of a call whose products find their rows themselves
constexpr int kSmall = 512;             // rows from which on workgroups have 64 (32 where ranks are many) and 32 rows in place of 16
constexpr int kWindow = 1 << 13;        // the most rows of one set of launches

// Rows order[first] .. of one adapter (-1: rows of none); count 0: nothing.
struct Item {
    int id, first, count, unused;
};

// What the launches of a window share, in the workspace
struct Lists {
    Item *in, *out;                     // for shrink and for expand
    int* order;
};

constexpr int rows_in(int64_t m, int64_t r) { return m < kSmall ? 16 : r > 64 ? 32 : 64; }

// T threads with U rows each, all ids at once.  `lds`: four numbers an adapter (and as many for none), kGroupBytes in front.  Items of 2^in_shift and
// 2^out_shift rows, in_most and out_most of them (those behind the last: nothing).
constexpr int kGroupBytes = 3 * 16 * 4;
constexpr int group_lds(int adapters) { return kGroupBytes + (4 * (adapters + 1) + 1) * 4; }

template <int T, int U>
__device__ __forceinline__ void group_rows(const LoraArgs& a, const Lists& lists, int in_shift, int out_shift, int in_most, int out_most, uint8_t* lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.adapters + 1;
    int *waves = reinterpret_cast<int*>(lds), *next = waves + 3 * 16, *begins = next + n, *in = begins + n + 1, *out = in + n;
    int id[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        id[u] = a.ids[min(u * T + (int)threadIdx.x, a.m - 1)];
    for (int i = threadIdx.x; i < n; i += T)
        next[i] = 0;
    __syncthreads();
    // Runs of one adapter: one addition a wave.
    const auto each = [&](auto take) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u * T >= a.m)
                break;
            const int row = u * T + (int)threadIdx.x, first = __builtin_amdgcn_readfirstlane(id[u]);
            if (__all(id[u] == first && row < a.m))
                take(row, first, true);
            else if (row < a.m)
                take(row, id[u], false);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        id[u] = id[u] >= 0 && id[u] < a.adapters ? id[u] : a.adapters;
    each([&](int, int of, bool run) {
        if (!run || lane == 0)
            atomicAdd(&next[of], run ? 64 : 1);
    });
    __syncthreads();
    const int per = (n + T - 1) / T, from = threadIdx.x * per, to = min(n, from + per);
    int sum[3] = {0, 0, 0}, all[3] = {0, 0, 0};                 // rows, items for shrink, items for expand in front of this thread's adapters; and of all
    const auto items = [](int rows, int shift) { return (rows + (1 << shift) - 1) >> shift; };
    for (int i = from; i < to; ++i) {
        sum[0] += next[i];
        sum[1] += i < a.adapters ? items(next[i], in_shift) : 0;
        sum[2] += items(next[i], out_shift);
    }
#pragma unroll
    for (int v = 0; v < 3; ++v) {
        int upto = sum[v];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int other = __shfl_up(upto, d);
            upto += lane >= d ? other : 0;
        }
        if (lane == 63)
            waves[v * 16 + wave] = upto;
        sum[v] = upto - sum[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < 3; ++v)
#pragma unroll
        for (int i = 0; i < T / 64; ++i) {
            sum[v] += i < wave ? waves[v * 16 + i] : 0;
            all[v] += waves[v * 16 + i];
        }
    for (int i = from; i < to; ++i) {
        const int rows = next[i];
        in[i] = sum[1];
        out[i] = sum[2];
        begins[i] = next[i] = sum[0];
        sum[0] += rows;
        sum[1] += i < a.adapters ? items(rows, in_shift) : 0;
        sum[2] += items(rows, out_shift);
    }
    if (threadIdx.x == 0)
        begins[n] = a.m;
    for (int i = all[1] + (int)threadIdx.x; i < in_most; i += T)
        lists.in[i] = Item{-1, 0, 0, 0};
    for (int i = all[2] + (int)threadIdx.x; i < out_most; i += T)
        lists.out[i] = Item{-1, 0, 0, 0};
    __syncthreads();
    each([&](int row, int of, bool run) {
        int place = !run || lane == 0 ? atomicAdd(&next[of], run ? 64 : 1) : 0;
        if (run)
            place = __builtin_amdgcn_readfirstlane(place) + lane;
        lists.order[place] = row;
        // the rows that come to an item's first place write it
        const int at = place - begins[of], left = begins[of + 1] - place, owner = of < a.adapters ? of : -1;
        if (owner >= 0 && (at & ((1 << in_shift) - 1)) == 0)
            lists.in[in[of] + (at >> in_shift)] = Item{owner, place, min(1 << in_shift, left), 0};
        if ((at & ((1 << out_shift) - 1)) == 0)
            lists.out[out[of] + (at >> out_shift)] = Item{owner, place, min(1 << out_shift, left), 0};
    });
}

__global__ __launch_bounds__(1024) void lora_group_kernel(LoraArgs a, Lists lists, int in_shift, int in_most, int out_most)
{
    extern __shared__ __align__(16) uint8_t smem[];
    group_rows<1024, kWindow / 1024>(a, lists, in_shift, 5, in_most, out_most, smem);
}

__global__ __launch_bounds__(512) void lora_group_few_kernel(LoraArgs a, Lists lists, int in_most, int out_most)
{
    extern __shared__ __align__(16) uint8_t smem[];
    group_rows<512, 1>(a, lists, 4, 4, in_most, out_most, smem);
}

// The rows of a workgroup of a product into `rows`, in the order of the call or the list; their adapter; how many they are.  Listed: item w.  Else: w has the
// adapter of that number, or where there are more adapters than rows, of the row of that number if it is the adapter's first; the number behind
// the last adapter (or row) has the rows of none.
constexpr int kListBytes = kAlone * 4;
template <bool kListed>
__device__ __forceinline__ int find(const LoraArgs& a, const Item* items, const int* order, int w, int* rows, int& cur)
{
    int count = 0;
    if constexpr (kListed) {
        const Item item = items[w];
        cur = item.id;
        count = item.count;
        if ((int)threadIdx.x < count)
            rows[threadIdx.x] = order[item.first + threadIdx.x];
    } else {
        const int lane = threadIdx.x & 63, most = min(a.adapters, a.m);
        const bool by_row = a.adapters > a.m;
        int id[kAlone / 64];
#pragma unroll
        for (int u = 0; u < kAlone / 64; ++u) {
            id[u] = a.ids[min(u * 64 + lane, a.m - 1)];
            id[u] = u * 64 + lane >= a.m ? -2 : id[u] >= 0 && id[u] < a.adapters ? id[u] : -1;
        }
        cur = w == most ? -1 : w;
        if (by_row && w < most) {
#pragma unroll
            for (int u = 0; u < kAlone / 64; ++u)
                if (w >> 6 == u)
                    cur = __builtin_amdgcn_readlane(id[u], w & 63);
            if (cur < 0)
                return 0;
        }
#pragma unroll
        for (int u = 0; u < kAlone / 64; ++u) {
            const uint64_t mine = __ballot(id[u] == cur);
            if (by_row && w < most && count == 0 && mine && u * 64 + __builtin_ctzll(mine) != w)
                return 0;
            if (id[u] == cur)                                   // (every wave writes the same)
                rows[count + __builtin_popcountll(mine & ((1ull << lane) - 1))] = u * 64 + lane;
            count += __builtin_popcountll(mine);
        }
    }
    if (count)
        __syncthreads();
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

template <int RT, int RG, int WK, int D, bool kListed>
__global__ __launch_bounds__(512) void lora_shrink_kernel(LoraArgs a, Lists lists, int k_part, int owners, int share)
{
    constexpr int kPhase = phase_of(WK), kBuf = shrink_buffer(RT, RG, WK), kRow = 64 * WK, kChunks = kRow / 16;
    constexpr int WR = 8 / WK, MR = RT / WR, C = (RT + RG) * WK / 8, kX = RT * WK;           // loads of a wave, KiB of x
    static_assert(MR * WR == RT && C * 8 == (RT + RG) * WK && kX % 8 == 0, "whole tiles and loads a wave");
    extern __shared__ __align__(16) uint8_t all_lds[];
    int* list = reinterpret_cast<int*>(all_lds);
    uint8_t* smem = all_lds + kListBytes;
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wk = wave % WK, wr = wave / WK;
    // Neighbouring workgroups have the parts of K in turn: a part of A's columns stays with the dies that have it.
    const int part = (int)(blockIdx.x % a.splits);
    const int k0 = part * k_part, k1 = min(a.k, k0 + k_part), phases = (k1 - k0 + kPhase - 1) / kPhase;
    const uint32_t lds_at = lds_address(smem);
    const int w = (int)(blockIdx.x / a.splits);
    int cur;
    const int count = find<kListed>(a, lists.in, lists.order, kListed ? w : w % owners, list, cur);
    for (int first = kListed ? 0 : w / owners * 16; first < count; first += share * 16) {
        const auto row_of = [&](int j) { return first + j < count ? list[first + j] : -1; };
        const u32x4_t rx = words16(a.x, (int64_t)a.m * a.ldx * 2), ra = words16(a.a + (int64_t)cur * a.r * a.k, (int64_t)a.r * a.k * 2);
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
                *reinterpret_cast<f32x4_t*>(a.part + ((int64_t)part * a.m + row) * a.r + rank) = sum;
        }
        if constexpr (kListed)
            return;
        __syncthreads();                                        // (the sums have been read)
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
        // cut off, not rounded: the largest numbers stay finite.  A number of few bits is cut below itself, so that the lower part of none but 0 is 0:
        // that would make NaN of an infinity of B.  (Infinity itself: the largest number and infinity; NaN stays in the lower part.)
        auto cut = [](float v) { return (__float_as_uint(v) - (v != 0.f)) >> 16; };
        const uint32_t upper[2] = {cut(t[e]), cut(t[e + 1])};
        o[e >> 1] = upper[0] | upper[1] << 16;
        o[2 + (e >> 1)] = f32_to_bf16_rne2(t[e] - bf16_bits_to_f32(upper[0]), t[e + 1] - bf16_bits_to_f32(upper[1]));
    }
    return o;
}

// t of every row in place of its first part, eight upper numbers and eight lower ones of a thread's eight ranks, so that the
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

// Below 512 rows: grid x 256 outputs, y the workgroups of those.
template <int KC, bool kListed>
__global__ __launch_bounds__(256, 4) void lora_expand_few_kernel(LoraArgs a, Lists lists, int owners, int share)
{
    extern __shared__ __align__(16) uint8_t smem[];
    int* list = reinterpret_cast<int*>(smem);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Expand<KC> e{a, smem + kListBytes, (int)threadIdx.x & 63, wave};
    int cur;
    const int w = (int)blockIdx.y, count = find<kListed>(a, lists.out, lists.order, kListed ? w : w % owners, list, cur);
    int first = kListed ? 0 : w / owners * 16;
    if (first >= count || (cur < 0 && a.base == a.y))
        return;
    const int n0 = ((int)blockIdx.x * 4 + wave) * 64, own = expand_t(KC) + wave * (1024 * KC);
    if (cur >= 0)
        e.fetch(lds_address(e.smem) + own, cur, n0);            // (B's rows stay for all of the adapter's)
    const float scale = a.scales && cur >= 0 ? a.scales[cur] : 1.f;
    const auto base = e.rows_of(a.base, a.ldb, a.m), y = e.rows_of(a.y, a.ldy, a.m);
    for (bool next = false; first < count; first += share * 16, next = true) {
        const auto row_of = [&](int j) { return first + j < count ? list[first + j] : -1; };
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

// Grid x: `walks` times 256 outputs, those of an item's rows side by side, then the next item's (a piece of B stays with a die).
template <int KC, int RT>
__global__ __launch_bounds__(256, KC == 16 ? 2 : 3) void lora_expand_kernel(LoraArgs a, Lists lists, int walks, int chunks)
{
    extern __shared__ __align__(16) uint8_t smem[];
    int* list = reinterpret_cast<int*>(smem);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Expand<KC> e{a, smem + kListBytes, (int)threadIdx.x & 63, wave};
    int cur;
    const int count = find<true>(a, lists.out, lists.order, (int)(blockIdx.x / chunks), list, cur);
    if (count == 0 || (cur < 0 && a.base == a.y))
        return;
    const int own = wave * (1024 * KC);
    const auto output = [&](int walk) { return (((int)(blockIdx.x % chunks) * walks + walk) * 4 + wave) * 64; };
    const auto base = e.rows_of(a.base, a.ldb, a.m), y = e.rows_of(a.y, a.ldy, a.m);
    u32x4_t v[RT][2], out[RT][2];
    int row[RT], from[RT], to[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        row[i] = 16 * i + (e.lane & 15) < count ? list[16 * i + (e.lane & 15)] : -1;
        from[i] = e.offset(row[i], a.ldb);
        to[i] = e.offset(row[i], a.ldy);
    }
    if (cur < 0) {                                              // rows of no adapter: the base as it is
        for (int walk = 0; walk < walks; ++walk) {
            e.load(v, base, output(walk), from);
            e.store(v, y, output(walk), to);
        }
        return;
    }
    e.fetch(lds_address(e.smem) + own, cur, output(0));
    e.load(v, base, output(0), from);
    const auto sums = __builtin_amdgcn_make_buffer_rsrc(a.part, 0, a.m * a.r * 4, 0x00020000);
    bf16x8_t t[RT][KC / 4][2];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int q = 0; q < KC / 4; ++q)
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                const int rank = 32 * q + 8 * (e.lane >> 4);
                t[i][q][part] = __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(sums, rank < a.r && row[i] >= 0 ? (row[i] * a.r + rank + 4 * part) * 4 : kOob, 0, 0));
            }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // A wave goes alone: the next outputs' rows of B and base are on their way before this walk's outputs leave, and the wait for them does not wait for
    // the stores.
    for (int walk = 0; walk < walks; ++walk) {
        e.product(out, v, e.smem + own, [&](int i, int q, int part) { return t[i][q][part]; });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (the wave's part has been read)
        if (walk + 1 < walks) {
            e.fetch(lds_address(e.smem) + own, cur, output(walk + 1));
            e.load(v, base, output(walk + 1), from);
        }
        e.store(out, y, output(walk), to);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * RT) : "memory");
    }
}

// The rows of one set of launches: lists are made by one workgroup, offsets into x, base and y have 31 bits, and a grid less than 2^32 threads.
int64_t window(const LoraArgs& a)
{
    return min(min((int64_t)min(a.m, kWindow), ((int64_t)1 << 29) / max(a.ldx, max(a.ldb, a.ldy))), max(((int64_t)1 << 31) / a.n, (int64_t)64));
}

// The launches of one window: RT tiles of sixteen rows and RG of ranks in shrink, ET tiles of rows in expand; kListed: with the sort in front.
template <int RT, int RG, int WK, int D, int ET, bool kListed>
hipError_t launch(const LoraArgs& a, hipStream_t stream)
{
    constexpr int KC = RG <= 2 ? 4 : RG <= 4 ? 8 : 16;
    constexpr bool kFew = ET == 1;
    constexpr int expand_bytes = 4 * 1024 * KC + (kFew ? expand_t(KC) : 0) + kListBytes, shrink_bytes = shrink_lds(RT, RG, WK, D) + kListBytes;
    static LdsLimit group, shrink, expand;
    hipError_t e = shrink.raise(reinterpret_cast<const void*>(lora_shrink_kernel<RT, RG, WK, D, kListed>), shrink_bytes);
    const void *first, *second;
    if constexpr (kFew) {
        first = reinterpret_cast<const void*>(lora_group_few_kernel);
        second = reinterpret_cast<const void*>(lora_expand_few_kernel<KC, kListed>);
    } else {
        first = reinterpret_cast<const void*>(lora_group_kernel);
        second = reinterpret_cast<const void*>(lora_expand_kernel<KC, ET>);
    }
    if (e == hipSuccess)
        e = expand.raise(second, expand_bytes);
    if (kListed && e == hipSuccess)
        e = group.raise(first, group_lds(kMostAdapters));
    if (e != hipSuccess)
        return e;
    Lists lists = {};
    lists.in = reinterpret_cast<Item*>(a.part + (int64_t)a.splits * a.m * a.r);
    lists.out = lists.in + a.m;
    lists.order = reinterpret_cast<int*>(lists.out + a.m);
    // An adapter's last item may have fewer rows than the others, and so may that of the rows of none.  Without lists, two workgroups an adapter
    // at least: 128 rows of one among 60, 4096 -> 4096, rank 16, 17.2 us for 25.5; 12.2 for 11.4 where the rows are mixed.
    const int owners = min(a.adapters, a.m), tiles = (a.m + 15) / 16, share = min(tiles, max(2, (2 * tiles + owners - 1) / owners));
    const int in = kListed ? min(a.m, a.m / (16 * RT) + owners) : owners * share;
    const int out = kListed ? min(a.m, a.m / (16 * ET) + owners + 1) : (owners + 1) * share;
    if constexpr (kListed && kFew)
        lora_group_few_kernel<<<1, 512, group_lds(a.adapters), stream>>>(a, lists, in, out);
    else if constexpr (kListed)
        lora_group_kernel<<<1, 1024, group_lds(a.adapters), stream>>>(a, lists, RT == 4 ? 6 : 5, in, out);
    const int k_part = ((a.k + a.splits - 1) / a.splits + phase_of(WK) - 1) / phase_of(WK) * phase_of(WK);
    lora_shrink_kernel<RT, RG, WK, D, kListed><<<in * a.splits, 512, shrink_bytes, stream>>>(a, lists, k_part, owners, share);
    if constexpr (kFew) {
        lora_expand_few_kernel<KC, kListed><<<dim3((a.n + 255) / 256, out), 256, expand_bytes, stream>>>(a, lists, owners + 1, share);
    } else {
        lora_sum_kernel<<<(a.m * (a.r / 8) + 255) / 256, 256, 0, stream>>>(a);
        const int64_t pieces = ((int64_t)a.m + 16 * ET - 1) / (16 * ET) * ((a.n + 255) / 256);
        const int walks = (int)min(max(pieces / 768, (int64_t)1), (int64_t)4), chunks = (a.n + 256 * walks - 1) / (256 * walks);
        lora_expand_kernel<KC, ET><<<out * chunks, 256, expand_bytes, stream>>>(a, lists, walks, chunks);
    }
    return hipGetLastError();
}

template <int RG, int D>
hipError_t launch_few(const LoraArgs& a, hipStream_t stream)
{
    return a.m <= kAlone ? launch<1, RG, 8, D, 1, false>(a, stream) : launch<1, RG, 8, D, 1, true>(a, stream);
}

int splits_of(int64_t m, int64_t k, int64_t r)
{
    const int64_t tiles = (m + rows_in(m, r) - 1) / rows_in(m, r), phase = phase_of(m < kSmall ? 8 : 4), most = (k + phase - 1) / phase;
    if (m < kSmall)
        return (int)(most < kLoraSplits ? most : kLoraSplits);
    // A power of two, so that neighbouring workgroups' parts fall on the same of the eight dies each time: six parts in place of four are longer (5003 rows
    // of 4096 -> 4096, rank 128: 66 us in four, 69 in six; 6000 of 11008 -> 4096: 97 and 105).
    int s = kLoraSplits;
    while (s > 1 && (s > most || s * tiles > 1024))
        s /= 2;
    return s;
}

}  // namespace

size_t lora_workspace(int64_t m, int64_t k, int64_t r)
{
    m = m < kWindow ? m : kWindow;
    // (a window that far strides make smaller may have more parts, but not of more than 1024 workgroups' rows)
    const int64_t rows = m < kSmall ? splits_of(m, k, r) * m : min(kLoraSplits * m, max(m, (int64_t)1024 * rows_in(m, r)));
    return (size_t)(rows * r) * 4 + (m > kAlone ? (size_t)m * (2 * sizeof(Item) + 4) : 0);
}

hipError_t launch_lora(const LoraArgs& whole, const DeviceInfo&, hipStream_t stream)
{
    const int64_t most = window(whole);
    const int ranks = (whole.r + 15) / 16;
    for (int64_t at = 0; at < whole.m; at += most) {
        LoraArgs a = whole;
        a.m = (int)min(whole.m - at, most);
        a.x += at * a.ldx;
        a.ids += at;
        a.base = a.base ? a.base + at * a.ldb : nullptr;
        a.y += at * a.ldy;
        a.splits = splits_of(a.m, a.k, a.r);
        hipError_t e;
        if (a.m < kSmall)
            e = ranks <= 1   ? launch_few<1, 4>(a, stream)
                : ranks <= 2 ? launch_few<2, 3>(a, stream)
                : ranks <= 4 ? launch_few<4, 2>(a, stream)
                             : launch_few<8, 2>(a, stream);
        else
            e = ranks <= 2   ? launch<4, 2, 4, 2, 2, true>(a, stream)
                : ranks <= 4 ? launch<4, 4, 2, 3, 2, true>(a, stream)
                             : launch<2, 8, 4, 2, 2, true>(a, stream);
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

}  // namespace mxfp4
