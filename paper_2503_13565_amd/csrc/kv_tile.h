// What the attention kernels over a paged MXFP4 cache share: how the work of a batch is cut into workgroups, and how 32
// cached tokens become operands of the matrix instructions in registers.
#pragma once

#include "common.h"
#include "kv.h"

namespace mxfp4 {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Maximum over the four lanes that hold one query's scores (l, l + 16, l + 32, l + 48), in all of them.
__device__ __forceinline__ float max_of_three(float a, float b, float c)
{
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);      // (one instruction; a NaN is the maximum)
}
__device__ __forceinline__ float max_of_rows(float v)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
    v = __builtin_elementwise_maximum(__int_as_float(p[0]), __int_as_float(p[1]));
    p = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
    return __builtin_elementwise_maximum(__int_as_float(p[0]), __int_as_float(p[1]));
}
__device__ __forceinline__ float max_of_wave(float v)
{
    v = fmaxf(v, dpp_f32<0xB1>(v));
    v = fmaxf(v, dpp_f32<0x4E>(v));
    v = fmaxf(v, dpp_f32<0x141>(v));
    return max_of_rows(fmaxf(v, dpp_f32<0x140>(v)));
}
__device__ __forceinline__ float sum_of_rows(float v)
{
    auto p = __builtin_amdgcn_permlane16_swap(__float_as_int(v), __float_as_int(v), false, false);
    v = __int_as_float(p[0]) + __int_as_float(p[1]);
    p = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
    return __int_as_float(p[0]) + __int_as_float(p[1]);
}

// One workgroup's share: key/value head h, query tile `tile` and part s of S of sequence b.
struct KvItem {
    int b, h, tile, s, S;
    int slot0, slots;                // the partial result of part 0, and the step from one part to the next
    int n, len, first;               // new tokens, cached tokens, first packed token of the sequence
};

// A row's new tokens, its length (both held to what the tables can hold) and where its keys begin to count.
struct KvRow {
    int n, len, first, lo;
    bool down;                       // its starts descend
};
__device__ __forceinline__ KvRow kv_row(const KvAttend& a, int b)
{
    KvRow r;
    if (a.b.starts) {
        const int from = a.b.starts[b], to = a.b.starts[b + 1];
        r.first = min(max(from, 0), a.b.tokens);
        r.n = min(max(to, r.first), a.b.tokens) - r.first;
        r.down = to < from;
    } else {
        r.first = b * a.b.per_row;
        r.n = a.b.per_row;
        r.down = false;
    }
    r.len = min(max(a.b.lens[b], 0), a.b.width << a.c.shift);
    r.lo = a.window > 0 ? max(0, min(r.len, r.len - r.n + 1 - a.window)) & ~31 : 0;
    return r;
}

// The cutting.  A sequence's range of keys counts in units of kUnit tokens; with U units in all (every head, every
// query tile) a part gets about L = U / target of them, so a row of n units has ceil(n / L) parts, and there are at most
// 2 target + (heads x tiles) workgroups.  Each finds its own share from the lengths, so that one launch fits any lengths, also those that
// change between replays of a graph, and sequences of different lengths load the device evenly.  Only rows of two parts or more need
// partial results: at most 4 target of them (U is summed in FP32, which all workgroups do alike; a few more for its rounding).
// What the parts aim for (us; 64 query heads on 8 of dim 128 where nothing else is said, 16 on 2 of dim 256 with four times the rows; both sides
// of every rule at six head sizes are in profiles/paged_cache_cutting.txt):
//   as they are  rows whose longest ends no later than parts would, the joining (`joint` units' time) with them; and starts that descend
//                somewhere: the rows then have more shares together than the launch has workgroups, and a row's parts would wait
//                for some that never come, with their counter above zero (56 rows of 4000 tokens: 54, 65 in parts; 60 of 8000: 102 and 113; dim
//                256: 140 and 166.  Without the joining's units the rule misses all of these; with twice as many a row of 1000 takes 10.7, not 9.2)
//   one round    with few rows of one length, the shortest parts that `target` workgroups hold at once (20 rows of 9000 tokens: 48, and 56 with a
//                workgroup's share each; 24 of 16000: 95 and 109; dim 256, 40 of 20000: 139 and 153; 16 of 32000: 108 and 110)
//   several      with many rows of different lengths, parts of half a workgroup's share, since parts of one length do not come out
//                (64 rows of 500 to 16384 tokens: 82, not 86; dim 192: 116, not 123; no more than 1 % at dims 32, 64 and 256)
//   short parts  (up to `brief` units) half of `target`, because joining costs more than it saves (4 rows of 16000 tokens: 22.7, not
//                24.4; 4 heads of dim 192: 30, not 43; `brief` of 32: one row of 131071 41, not 37)
//   a row alone  no more than the kKvJoin parts that are joined at a time, unless that leaves a part over four units (one row of 4000 tokens
//                11.0, 12.1 with two units, of 16000 15.0, 17.7 with eight); whole up to six units (500 tokens 8.3, 9.4 in parts; 1000 9.2,
//                11.0 whole)
constexpr int kKvJoin = 8;
template <int kUnit>
__device__ __forceinline__ bool kv_find(const KvAttend& a, int item, int tile_rows, int brief, int joint, KvItem* out)
{
    const int lane = threadIdx.x & 63;
    KvRow r0 = {0, 0, 0, 0, false};
    bool down = false;
    float all = 0.f, longest = 0.f, whole = 0.f;    // units, those of the longest row, rows of keys
    for (int base = 0; base < a.b.rows; base += 64) {
        float u = 0.f, t = 0.f;
        if (base + lane < a.b.rows) {
            const KvRow r = kv_row(a, base + lane);
            const float tiles = (float)((r.n * a.group + tile_rows - 1) / tile_rows), units = (float)max(1, (r.len - r.lo + kUnit - 1) / kUnit);
            u = tiles * units;
            t = tiles;
            longest = fmaxf(longest, tiles > 0.f ? units : 0.f);
            down |= r.down;
            if (base == 0)
                r0 = r;
        }
        all += wave_sum(u);
        whole += wave_sum(t);
    }
    longest = max_of_wave(longest);
    all *= (float)a.c.heads;
    whole *= (float)a.c.heads;
    const float target = (float)a.target, even = ceilf(all / target);
    float aim = even;
    if (__ballot(down) || fmaxf(longest, all / target + 0.5f * longest) <= 1.5f * all / target + (float)joint) {
        aim = 1e9f;
    } else if (2.f * whole <= target && longest * whole <= 1.05f * all && a.b.rows <= 64) {
        const int tiles = (r0.n * a.group + tile_rows - 1) / tile_rows * a.c.heads, units = max(1, (r0.len - r0.lo + kUnit - 1) / kUnit);
        for (int i = 0; i < 4; ++i) {
            aim = ceilf(even * (1.f + 0.25f * (float)i));
            const int parts = (units + (int)aim - 1) / (int)aim;
            if (wave_sum(lane < a.b.rows ? (float)tiles * (float)parts : 0.f) <= target)
                break;
        }
    } else if (even > (float)brief && longest * whole > 1.25f * all) {
        aim = ceilf(0.5f * even);
    }
    const int each = (int)fminf(fmaxf(aim, fminf(2.f * even, (float)brief)), 1e9f);
    int before = 0, slots = 0;
    for (int base = 0; base < a.b.rows; base += 64) {
        KvRow r = r0;
        int parts = 1, tiles = 0;
        if (base + lane < a.b.rows) {
            if (base)
                r = kv_row(a, base + lane);
            tiles = (r.n * a.group + tile_rows - 1) / tile_rows;
            const int units = max(1, (r.len - r.lo + kUnit - 1) / kUnit);
            const int mine = max(each, units <= 6 ? units : min((units + kKvJoin - 1) / kKvJoin, 4));
            parts = (units + mine - 1) / mine;
        }
        const int mine = tiles * parts * a.c.heads;
        const int upto = before + wave_scan(mine);
        const int slots_upto = slots + wave_scan(parts > 1 ? mine : 0);
        const uint64_t there = __ballot(upto > item);
        if (there) {
            const int at = __ffsll((unsigned long long)there) - 1;
            const int local = item - __builtin_amdgcn_readlane(upto - mine, at);
            const int S = __builtin_amdgcn_readlane(parts, at), T = __builtin_amdgcn_readlane(tiles, at);
            out->b = base + at;
            out->S = S;
            out->h = local % a.c.heads;                  // neighbouring workgroups: the heads, so that a head's tiles meet in one L2
            const int rest = local / a.c.heads;
            out->tile = T - 1 - rest % T;                // causal: the tiles with the most keys first
            out->s = rest / T;
            out->slots = T * a.c.heads;
            out->slot0 = __builtin_amdgcn_readlane(slots_upto - (parts > 1 ? mine : 0), at) + out->tile * a.c.heads + out->h;
            out->n = __builtin_amdgcn_readlane(r.n, at);
            out->len = __builtin_amdgcn_readlane(r.len, at);
            out->first = __builtin_amdgcn_readlane(r.first, at);
            return true;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
        slots = __builtin_amdgcn_readlane(slots_upto, 63);
    }
    return false;
}

// 32 tokens of one head as a wave loads them.  Keys: lane (r, g) = (lane % 16, lane / 16) has the NB dwords of tokens r and 16 + r
// that hold elements 8 NB g .. 8 NB (g + 1) - 1, which are its eight elements of each of NB products (the queries are laid out to
// match).  Values: lane (r, g) has tokens 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3, the tokens whose weights the same lane gets
// out of the score products; of each token elements kEl r .. kEl (r + 1) - 1 of every chunk of 16 kEl, so that
// the eight tokens of one element are an operand without any crossing of lanes.
// NB is 1, 2, 4 or 8; kPad: the head has fewer than 32 NB elements (96 of 128, 192 of 256), the lanes of the missing ones hold zeros.
template <int NB, bool kPad>
struct KvTile {
    static constexpr int kEl = NB >= 4 ? 8 : NB == 2 ? 4 : 2;            // elements of a chunk in one lane
    static constexpr int kChunk = 16 * kEl, kChunks = NB * 32 / kChunk;
    static constexpr int kBlocks = kChunk / 32;                          // scale blocks of a chunk
    static constexpr int kKs = NB == 8 ? 2 : 1;                          // scale blocks of a lane's key elements
    uint32_t k[2][NB];
    uint32_t v[2][4][kChunks];
    uint32_t vs[2][kPad ? 4 * kChunks : NB];                             // four tokens' bytes as they lie, or a byte each
    uint32_t ks[2][kKs];
    int page[2];                                                         // of the two halves; -1: not there (uniform)
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t* out, const uint8_t* p)
{
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4_t w = *reinterpret_cast<const u32x4_t*>(p + 4 * i);
            out[i] = w[0], out[i + 1] = w[1], out[i + 2] = w[2], out[i + 3] = w[3];
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const uint2 w = *reinterpret_cast<const uint2*>(p + 4 * i);
            out[i] = w.x, out[i + 1] = w.y;
        }
    } else {
        out[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}

// Page of each half of 32 tiles of a wave, `step` tiles apart: lane 2 i + half has tile i's.  -1 where the table names none.
template <int kStep>
__device__ __forceinline__ int kv_pages32(const KvAttend& a, int b, int len, int tile)
{
    const int lane = threadIdx.x & 63;
    const int at = (tile + (lane >> 1) * kStep) * 32 + (lane & 1) * 16;
    return at < len ? kv_page(a.b.table, a.b.ldt, a.b.width, a.c.shift, a.c.pages, b, at) : -1;
}

template <int NB, bool kPad>
__device__ __forceinline__ void load_tile(KvTile<NB, kPad>& t, const KvView& c, int h, int token, int page0, int page1)
{
    typedef KvTile<NB, kPad> T;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    const int nb = kPad ? c.nb : NB;
    t.page[0] = page0;
    t.page[1] = page1;
#pragma unroll
    for (int a = 0; a < 2; ++a) {
        const int page = max(t.page[a], 0);              // a half that is not there is read from page 0 and left out
        const int slot = (h << c.shift) + ((token + 16 * a) & ((1 << c.shift) - 1));
        const int64_t at_q = (int64_t)page * c.psq + (int64_t)slot * (16 * nb), at_s = (int64_t)page * c.pss + (int64_t)slot * nb;
        const uint8_t *kq = c.kq + at_q, *vq = c.vq + at_q, *ks = c.ks + at_s, *vs = c.vs + at_s;
#pragma unroll
        for (int b = 0; b < T::kKs; ++b) {
            const int block = T::kKs * g + b;            // (NB = 1, 2: a quarter, a half of a block in a lane)
            const bool has = !kPad || block < nb;
            t.ks[a][b] = 0;
            if constexpr (NB >= 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    t.k[a][4 * b + i] = 0;
                if (has)
                    load_words<4>(&t.k[a][4 * b], kq + (uint32_t)((r * nb + block) * 16));
            } else {
                load_words<NB>(t.k[a], kq + (uint32_t)((r * 16 + 4 * g) * NB));
            }
            if (has)
                t.ks[a][b] = ks[(uint32_t)(r * nb + (NB >= 4 ? block : (NB * g) >> 2))];
        }
        if constexpr (!kPad)
            load_words<NB>(t.vs[a], vs + (uint32_t)(4 * g * NB));
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int ch = 0; ch < T::kChunks; ++ch) {
                // (32-bit offsets without a sign: the base stays in scalar registers)
                const uint8_t* p = vq + (uint32_t)((4 * g + i) * 16 * nb + ch * (T::kChunk / 2) + r * (T::kEl / 2));
                if constexpr (kPad) {
                    const int block = ch * T::kBlocks + ((r * T::kEl) >> 5);
                    t.v[a][i][ch] = t.vs[a][i * T::kChunks + ch] = 0;
                    if (block < nb) {
                        t.v[a][i][ch] = *reinterpret_cast<const uint32_t*>(p);
                        t.vs[a][i * T::kChunks + ch] = vs[(uint32_t)((4 * g + i) * nb + block)];
                    }
                } else {
                    t.v[a][i][ch] = T::kEl == 8 ? *reinterpret_cast<const uint32_t*>(p)
                                                : T::kEl == 4 ? (uint32_t)*reinterpret_cast<const uint16_t*>(p) : (uint32_t)*p;
                }
            }
    }
}

// Eight elements of a dword of codes as BF16; byte 255 of the scale is NaN to the convert, 0 is 2^-127.
__device__ __forceinline__ bf16x8_t eight_of(uint32_t w, uint32_t byte)
{
    const float s = __uint_as_float(byte << 23);
    u32x4_t x;
    x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
    x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
    x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
    x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
    return __builtin_bit_cast(bf16x8_t, x);
}

// The lane's eight key elements of product j of half a.
template <int NB, bool kPad>
__device__ __forceinline__ bf16x8_t key_operand(const KvTile<NB, kPad>& t, int a, int j)
{
    return eight_of(t.k[a][j], t.ks[a][KvTile<NB, kPad>::kKs == 2 ? j >> 2 : 0]);
}

// The scale byte of token i of half a, chunk ch, in this lane; and the byte made 0 (2^-127: zero codes are zeros with any but NaN).
template <int NB, bool kPad>
__device__ __forceinline__ int value_scale_shift(int i, int ch)
{
    typedef KvTile<NB, kPad> T;
    return 8 * ((i * NB + ch * T::kBlocks) & 3) + 8 * (((threadIdx.x & 15) * T::kEl) >> 5);
}
template <int NB, bool kPad>
__device__ __forceinline__ uint32_t value_scale(const KvTile<NB, kPad>& t, int a, int i, int ch)
{
    typedef KvTile<NB, kPad> T;
    if constexpr (kPad)
        return t.vs[a][i * T::kChunks + ch];
    else
        return __builtin_amdgcn_ubfe(t.vs[a][(i * NB + ch * T::kBlocks) >> 2], value_scale_shift<NB, kPad>(i, ch), 8);
}
template <int NB, bool kPad>
__device__ __forceinline__ void clear_value(KvTile<NB, kPad>& t, int a, int i, int ch)
{
    typedef KvTile<NB, kPad> T;
    t.v[a][i][ch] = 0;
    if constexpr (kPad)
        t.vs[a][i * T::kChunks + ch] = 0;
    else
        t.vs[a][(i * NB + ch * T::kBlocks) >> 2] &= ~(0xFFu << value_scale_shift<NB, kPad>(i, ch));
}

// The lane's operands of one chunk of the values: x[e] holds its eight tokens of element kEl r + e.  Two tokens' converts
// give pairs of elements; a byte permute each makes pairs of tokens of them (the scale differs from token to token, so the
// tokens cannot be paired in front of the convert).
template <int NB, bool kPad>
__device__ __forceinline__ void value_operands(const KvTile<NB, kPad>& t, int ch, bf16x8_t* x)
{
    typedef KvTile<NB, kPad> T;
    u32x4_t y[T::kEl];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const int a = m >> 1, i = (m & 1) * 2;
        const float s0 = __uint_as_float(value_scale(t, a, i, ch) << 23), s1 = __uint_as_float(value_scale(t, a, i + 1, ch) << 23);
        const uint32_t w0 = t.v[a][i][ch], w1 = t.v[a][i + 1][ch];
#define MXFP4_PAIR(e)                                                                                                     \
    if constexpr (2 * e < T::kEl) {                                                                                       \
        const uint32_t c0 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w0, s0, e));           \
        const uint32_t c1 = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w1, s1, e));           \
        y[2 * e][m] = __builtin_amdgcn_perm(c1, c0, 0x05040100u);                                                         \
        y[2 * e + 1][m] = __builtin_amdgcn_perm(c1, c0, 0x07060302u);                                                     \
    }
        MXFP4_PAIR(0)
        MXFP4_PAIR(1)
        MXFP4_PAIR(2)
        MXFP4_PAIR(3)
#undef MXFP4_PAIR
    }
#pragma unroll
    for (int e = 0; e < T::kEl; ++e)
        x[e] = __builtin_bit_cast(bf16x8_t, y[e]);
}

// What the queries of a stretch see: query at position p (kNobody: no query) sees position j.
constexpr int kNobody = -0x40000000;
struct KvSight {
    int base, window;                // position of the sequence's first new token; 0: all before
    bool causal, tree;
    __device__ __forceinline__ bool sees(int p, uint64_t word, int j) const
    {
        bool ok = p != kNobody && (!causal || j <= p) && (window == 0 || j > p - window);
        if (tree && j >= base)
            ok = ok && j - base < 64 && ((word >> (j - base)) & 1);
        return ok;
    }
    __device__ __forceinline__ uint64_t word(const KvAttend& a, const KvItem& it, int p) const
    {
        return tree && p != kNobody ? a.tree[it.first + p - base] : 0;
    }
};

// Where part s of S begins among n.
__device__ __forceinline__ int part_begin(int n, int s, int S)
{
    const int each = n / S;
    return s * each + min(s, n - each * S);
}

// One query tile's scores of 32 tokens (lane (query, g): tokens 4 g + i of either half) become weights, the right operand of the
// values' product.  The running maximum m and the sums move with it: o of the values, l of the weights as the values' product has
// them, rounded (in all four registers, as the matrix instruction leaves it), and, if it is wanted, `exact` of the lane's weights
// as they are, for the logarithm, in which a single weight's rounding would show.  A NaN score makes `top` NaN (the maximum here is
// the one that carries it on), which moves nothing, and a NaN weight, which makes the query's sums NaN.
template <int kSums>
__device__ __forceinline__ bf16x8_t softmax_step(f32x4_t* s, float scale, bool wanted, float* m, f32x4_t* l, float* exact, f32x4_t* o)
{
    float top = max_of_three(max_of_three(max_of_three(s[0][0], s[0][1], s[0][2]), s[0][3], s[1][0]), s[1][1], s[1][2]);
    top = max_of_rows(max_of_three(top, s[1][3], s[1][3]));
    // The sums move to a new maximum only when it is 2^8 above the old one: the weights then stay below 2^8, which FP32 sums and
    // BF16 weights hold as well as weights up to 1.  (The first maximum is infinitely far above none.)
    // A weight's exponent is (s - m) scale, with the difference first: it is exact next to the maximum.  s scale - m scale is one operation
    // less, and the rounding of its second product stays in it: 2^-15 at most while that product is below 2^10, but a weight of 2^128 where
    // it is 2^31.  Up to dim 128 (vector-bound with many queries: 303 us for 5001 tokens of a prompt, 310 with eight more operations) it is
    // taken below 2^10, and past that the maximum leaves the scores in the rescaling's branch, so that the usual tile has no more blocks
    // than before; the larger heads, where that costs 1 to 7 % and the operations nothing, take the difference always.
    constexpr bool kFused = kSums <= 8;
    float off = kFused && *m != -INFINITY ? -*m * scale : 0.f;
    if (__ballot((top - *m) * scale > 8.f || fabsf(off) > 1024.f)) {
        const float now = top > *m ? top : *m;
        const float f = now == -INFINITY ? 1.f : exp2f((*m - now) * scale);
        *m = now;
        *l *= f;
        *exact *= f;
#pragma unroll
        for (int e = 0; e < kSums; ++e)
            o[e] *= f;
        if constexpr (kFused) {
            off = now == -INFINITY ? 0.f : -now * scale;
            const float first = fabsf(off) > 1024.f ? now : 0.f;
            off = fabsf(off) > 1024.f ? 0.f : off;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[i >> 2][i & 3] -= first;
        }
    }
    const float base = *m == -INFINITY ? 0.f : *m;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w[i] = __builtin_amdgcn_exp2f(kFused ? fmaf(s[i >> 2][i & 3], scale, off) : (s[i >> 2][i & 3] - base) * scale);
    // rounded to BF16 (the type of the values' product; half a step, 2^-8 of a weight at most, and the weights' errors average out: the result is
    // off by 2.0e-3 to 2.3e-3 of its norm, its own rounding alone by 1.65e-3).  What the rounding leaves of a weight as a second BF16 operand
    // takes that back to 1.65e-3 and costs every row a second product: one token over 131071 39.7 us, not 38.4, 64 rows of 500 to 16384 88.5,
    // not 85.4, 16 rows of 8000 38.4, not 33.9, pieces and prompts, which the vector unit bounds, 79.5, not 69 and 357, not 304.
    const bf16x8_t p = __builtin_bit_cast(bf16x8_t, (u32x4_t{f32_to_bf16_rne2(w[0], w[1]), f32_to_bf16_rne2(w[2], w[3]),
                                                             f32_to_bf16_rne2(w[4], w[5]), f32_to_bf16_rne2(w[6], w[7])}));
    if (wanted)
        *exact += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    // Their sum by one product with ones: the matrix pipe has room, the vector unit has not.
    const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, (u32x4_t{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u}));
    *l = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, p, *l, 0, 0, 0);
    return p;
}

// Values that are no numbers in a tile that not every query sees whole: all of a block of scale byte 255 (NaN), and infinities, codes
// of 2 and more under byte 254, of 4 and more under 253 (no cast gives them, a cache may be filled otherwise).  0 times them is NaN, so they
// leave the tile, and each query that sees one gets it by products of ones in the places of what is odd and of what the queries
// see: `all` counts what a query sees, `sum` the infinities with their signs, so that sum = all says +infinity, sum = -all -infinity, and
// anything else NaN.
constexpr uint32_t kOddScale = 253;
__device__ __forceinline__ uint32_t infinite_codes(uint32_t w, uint32_t byte)            // a bit for each element
{
    return (byte == 254 ? w >> 2 : byte == 253 ? (w >> 2) & (w >> 1) : 0u) & 0x11111111u;
}
template <int NB, bool kPad>
__device__ __forceinline__ void drop_odd_values(KvTile<NB, kPad>& t)
{
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int ch = 0; ch < KvTile<NB, kPad>::kChunks; ++ch) {
            const uint32_t byte = value_scale(t, k >> 2, k & 3, ch);
            t.v[k >> 2][k & 3][ch] &= ~(15 * infinite_codes(t.v[k >> 2][k & 3][ch], byte));
            if (byte == 255)
                clear_value(t, k >> 2, k & 3, ch);
        }
}
template <int QT, int kSums, int NB, bool kPad>
__device__ __forceinline__ void add_odd_values(const KvTile<NB, kPad>& t, int ch, const bf16x8_t* seen, f32x4_t (*o)[kSums])
{
    typedef KvTile<NB, kPad> T;
    uint32_t odd[8];                                     // of each token: for each element a bit "odd", one "infinite", one "negative"
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const uint32_t w = t.v[k >> 2][k & 3][ch], byte = value_scale(t, k >> 2, k & 3, ch), inf = infinite_codes(w, byte);
        odd[k] = byte == 255 ? 0x11111111u : 3 * inf | (w >> 3 & inf) << 2;
    }
#pragma unroll 1
    for (int e = 0; e < T::kEl; ++e) {                   // (rare: the elements take turns in one copy of the code)
        u32x4_t x, y;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const uint32_t n0 = odd[2 * m] >> (4 * e), n1 = odd[2 * m + 1] >> (4 * e);
            x[m] = (n0 & 1 ? 0x3F80u : 0u) | (n1 & 1 ? 0x3F800000u : 0u);
            y[m] = (n0 & 2 ? 0x3F80u | (n0 & 4) << 13 : 0u) | (n1 & 2 ? 0x3F800000u | (n1 & 4) << 29 : 0u);
        }
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
            const f32x4_t all = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), seen[qt], zero, 0, 0, 0);
            const f32x4_t sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, y), seen[qt], zero, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < T::kEl; ++k)
                if (k == e)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (all[i] > 0.f)
                            o[qt][ch * T::kEl + k][i] += __uint_as_float(sum[i] == all[i] ? 0x7F800000u : sum[i] == -all[i] ? 0xFF800000u : 0x7FC00000u);
        }
    }
}

// Stores and loads that all dies of the device see alike.
__device__ __forceinline__ void put_through(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float get_through(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

}  // namespace mxfp4
