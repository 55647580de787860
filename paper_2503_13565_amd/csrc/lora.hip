// Low-rank adapters of many requests beside a shared projection:  y[m] = base[m] + scale[i] * B_i (A_i x[m]),  i = ids[m].
//
// Two launches.  The first makes t = A_i x for every row: a workgroup has RT tiles of 16 rows and a part of K, its four waves share the
// part, and each of the tile's different adapters takes one walk, in which the tile's rows are the columns of
// v_mfma_f32_16x16x32_bf16 and 16 ranks its rows; only the rows of that adapter keep the result, so that what another
// request's adapter holds (NaN, infinities) never meets a row.  The parts' sums lie side by side in the workspace, FP32.
// The second adds them in order, scales them and splits them into two BF16 numbers (together 16 bits of t, so that t's rounding
// does not show beside that of y), and multiplies with B_i in the same way, the base added to the FP32 sums: one rounding.
#include "common.h"
#include "layer.h"

namespace mxfp4 {

namespace {

constexpr int kRanks = 128;             // the largest rank of a call

__device__ __forceinline__ bf16x8_t load8(const uint16_t* p) { return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4_t*>(p)); }

// Matrix instructions run with all lanes.  Where their result is used by some lanes only, the compiler may move them behind that
// condition, and the operands of the other lanes with it; this keeps them in front.
__device__ __forceinline__ void settle(f32x4_t& v) { asm volatile("" : "+v"(v)); }

// The adapter of each of the tile's 16 RT rows, in the lane of its number; -1: none.
__device__ __forceinline__ int tile_ids(const LoraArgs& a, int64_t m0, int rows, int lane)
{
    const int id = lane < rows ? a.ids[m0 + lane] : -1;
    return id >= 0 && id < a.adapters ? id : -1;
}

template <int RT, int RG>
__global__ __launch_bounds__(256) void lora_shrink_kernel(LoraArgs a, int k_part)
{
    __shared__ f32x4_t red[4][RT * RG][64];
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = (int64_t)blockIdx.x * (16 * RT);
    const int rows = (int)min((int64_t)16 * RT, a.m - m0);
    const int id = tile_ids(a, m0, rows, lane);
    const int k0 = (int)blockIdx.y * k_part, k1 = min(a.k, k0 + k_part);
    const int slots = gridDim.z;
    uint64_t todo = __ballot(id >= 0);
    for (int nth = 0; todo; ++nth) {
        const int cur = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
        const uint64_t mine = __ballot(id == cur);
        todo &= ~mine;
        if (nth % slots != (int)blockIdx.z)
            continue;
        f32x4_t acc[RT][RG] = {};
        for (int kk = k0 + wave * 32; kk < k1; kk += 128) {
            const int at = kk + lg * 8;                         // (k is a multiple of 8: a lane's eight are inside or outside)
            bf16x8_t w[RG], x[RT];
#pragma unroll
            for (int f = 0; f < RG; ++f) {
                const int rank = f * 16 + li;
                w[f] = bf16x8_t{};
                if (rank < a.r && at < k1)
                    w[f] = load8(a.a + ((int64_t)cur * a.r + rank) * a.k + at);
            }
#pragma unroll
            for (int f = 0; f < RT; ++f) {
                const int row = f * 16 + li;
                x[f] = bf16x8_t{};
                if (row < rows && at < k1)
                    x[f] = load8(a.x + (m0 + row) * a.ldx + at);
            }
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int f = 0; f < RG; ++f)
                    acc[i][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[f], x[i], acc[i][f], 0, 0, 0);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int f = 0; f < RG; ++f)
                red[wave][i * RG + f][lane] = acc[i][f];
        __syncthreads();
        for (int at = threadIdx.x; at < RT * RG * 64; at += 256) {
            const int f = at >> 6, l = at & 63, row = f / RG * 16 + (l & 15), rank = f % RG * 16 + 4 * (l >> 4);
            const f32x4_t sum = red[0][f][l] + red[1][f][l] + red[2][f][l] + red[3][f][l];
            if ((mine >> row & 1) && rank < a.r)
                *reinterpret_cast<f32x4_t*>(a.part + ((int64_t)blockIdx.y * a.m + m0 + row) * a.r + rank) = sum;
        }
    }
}

// A wave has 64 outputs of 16 RT rows.  Row i + 4 j (i < 4) of B's fragment f is output 16 j + 4 f + i, so that a lane ends with 16
// outputs side by side of its row.
template <int RT>
__global__ __launch_bounds__(256) void lora_expand_kernel(LoraArgs a)
{
    constexpr int kStride = kRanks + 8;                         // (16 bytes more than the ranks: rows start in different banks)
    __shared__ uint16_t hi[RT * 16][kStride], lo[RT * 16][kStride];
    const int lane = threadIdx.x & 63, li = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t m0 = (int64_t)blockIdx.x * (16 * RT);
    const int rows = (int)min((int64_t)16 * RT, a.m - m0);
    const int id = tile_ids(a, m0, rows, lane);
    const int n0 = ((int)blockIdx.y * 4 + wave) * 64;
    const int slots = gridDim.z;
    const int ranks = (a.r + 31) & ~31;

    for (int at = threadIdx.x; at < RT * 16 * (ranks / 4); at += 256) {
        const int row = at / (ranks / 4), rank = at % (ranks / 4) * 4;
        const int of = row < rows ? a.ids[m0 + row] : -1;
        f32x4_t t = {0.f, 0.f, 0.f, 0.f};
        if (of >= 0 && of < a.adapters && rank < a.r) {
            for (int p = 0; p < a.splits; ++p)
                t += *reinterpret_cast<const f32x4_t*>(a.part + ((int64_t)p * a.m + m0 + row) * a.r + rank);
            if (a.scales)
                t *= a.scales[of];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // cut off, not rounded: the largest numbers stay finite
            const uint16_t h = t[e] == t[e] ? (uint16_t)(__float_as_uint(t[e]) >> 16) : (uint16_t)0x7FC0;
            const float rest = t[e] - bf16_bits_to_f32(h);
            hi[row][rank + e] = h;
            lo[row][rank + e] = rest == rest ? f32_to_bf16_rne(rest) : 0;        // (an infinity leaves no rest)
        }
    }
    __syncthreads();

    auto store = [&](int64_t row, const f32x4_t* sum) {         // outputs n0 + 16 lg .. + 15 of a row
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int n = n0 + 16 * lg + 8 * half;
            if (n >= a.n)
                return;
            u32x4_t v = {0, 0, 0, 0};
            if (a.base)
                v = *reinterpret_cast<const u32x4_t*>(a.base + row * a.ldb + n);
            if (sum)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x4_t z = sum[2 * half + (e >> 1)];
                    v[e] = f32_to_bf16_rne2(bf16_bits_to_f32(v[e] & 0xFFFFu) + z[2 * (e & 1)],
                                            __uint_as_float(v[e] & 0xFFFF0000u) + z[2 * (e & 1) + 1]);
                }
            *reinterpret_cast<u32x4_t*>(a.y + row * a.ldy + n) = v;
        }
    };

    if (blockIdx.z == 0 && a.base != a.y)                       // rows of no adapter
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int row = i * 16 + li;
            if (__shfl(id, row) < 0 && row < rows)
                store(m0 + row, nullptr);
        }
    uint64_t todo = __ballot(id >= 0);
    for (int nth = 0; todo; ++nth) {
        const int cur = __builtin_amdgcn_readlane(id, __builtin_ctzll(todo));
        const uint64_t mine = __ballot(id == cur);
        todo &= ~mine;
        if (nth % slots != (int)blockIdx.z)
            continue;
        f32x4_t acc[RT][4] = {};
        for (int kk = 0; kk < a.r; kk += 32) {
            bf16x8_t w[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int n = n0 + 16 * (li >> 2) + 4 * f + (li & 3), rank = kk + 8 * lg;
                w[f] = bf16x8_t{};
                if (n < a.n && rank < a.r)
                    w[f] = load8(a.b + ((int64_t)cur * a.n + n) * a.r + rank);
            }
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const bf16x8_t th = load8(&hi[i * 16 + li][kk + 8 * lg]), tl = load8(&lo[i * 16 + li][kk + 8 * lg]);
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
            for (int f = 0; f < 4; ++f)
                settle(acc[i][f]);
#pragma unroll
        for (int i = 0; i < RT; ++i)
            if (mine >> (i * 16 + li) & 1)
                store(m0 + i * 16 + li, acc[i]);
    }
}

// A grid holds less than 2^32 threads, so very many rows are several pairs of launches.
template <int RT, int RG>
hipError_t launch(LoraArgs a, int slots, hipStream_t stream)
{
    const int k_part = ((a.k + a.splits - 1) / a.splits + 31) / 32 * 32;
    const int64_t chunks = (a.n + 255) / 256, most = ((int64_t)1 << 23) / (chunks * slots) * (RT * 16), all = a.m;
    for (int64_t at = 0; at < all; at += most) {
        LoraArgs b = a;
        b.m = (int)(all - at < most ? all - at : most);
        b.x += at * a.ldx;
        b.ids += at;
        b.base = a.base ? a.base + at * a.ldb : nullptr;
        b.y += at * a.ldy;
        const unsigned tiles = (unsigned)((b.m + RT * 16 - 1) / (RT * 16));
        lora_shrink_kernel<RT, RG><<<dim3(tiles, a.splits, slots), 256, 0, stream>>>(b, k_part);
        lora_expand_kernel<RT><<<dim3(tiles, (unsigned)chunks, slots), 256, 0, stream>>>(b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

constexpr bool wide(int64_t m) { return m >= 512; }

}  // namespace

int lora_splits(int64_t m, int64_t k, int64_t)
{
    const int64_t tiles = wide(m) ? (m + 63) / 64 : (m + 15) / 16;
    int64_t s = 512 / tiles;
    if (s > 8)
        s = 8;
    if (s > (k + 127) / 128)
        s = (k + 127) / 128;
    return s < 1 ? 1 : (int)s;
}

hipError_t launch_lora(const LoraArgs& a, const DeviceInfo&, hipStream_t stream)
{
    const int groups = (a.r + 15) / 16;
    if (wide(a.m)) {
        const int slots = a.adapters < 4 ? a.adapters : 4;
        return groups <= 1   ? launch<4, 1>(a, slots, stream)
               : groups <= 2 ? launch<4, 2>(a, slots, stream)
               : groups <= 4 ? launch<4, 4>(a, slots, stream)
                             : launch<4, 8>(a, slots, stream);
    }
    const int slots = a.adapters < 16 ? (a.adapters < a.m ? a.adapters : a.m) : (a.m < 16 ? a.m : 16);
    return groups <= 1   ? launch<1, 1>(a, slots, stream)
           : groups <= 2 ? launch<1, 2>(a, slots, stream)
           : groups <= 4 ? launch<1, 4>(a, slots, stream)
                         : launch<1, 8>(a, slots, stream);
}

}  // namespace mxfp4
