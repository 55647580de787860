// Attention over a paged MXFP4 cache for gfx950: drafting (one token), verifying (a draft or a draft tree), pieces of prompts and
// whole ones.
//
//   out[t][h] = sum_j p_j v_j / sum_j p_j,   p_j = exp(scale q[t][h] . k_j - m)
//
// in one pass over the keys with the running maximum m.  With few queries bound by HBM: 17/16 bytes per element of the head dimension
// and token (codes and scales of key and value); with many by the vector unit, whose converts and softmax steps and the matrix
// instructions take turns (5001 tokens of a prompt: vector 64 % of a SIMD's cycles, matrix 28 %).  The queries of all heads that share a
// key/value head, and all new tokens, are the 16 columns of v_mfma_f32_16x16x32_bf16 (QT times 16), so a cached token is read and decoded
// once for all of them:
//   scores   S^T[token][query]  = K . Q^T      keys are the left operand, decoded in registers (kv_tile.h)
//   values   O^T[element][query] += V^T . P^T   the scores leave the first product in the layout in which the second one takes
//                                               them as its right operand: no LDS and no crossing of lanes in the loop
#include <algorithm>

#include "kv_tile.h"

namespace mxfp4 {

template <int NB, int QT, bool kPad>
__global__ __launch_bounds__(256, NB <= 4 ? 2 : 1) void kv_attend_kernel(KvAttend a)
{
    typedef KvTile<NB, kPad> T;
    constexpr int NW = 4, kRows = 16 * QT, kEl = T::kEl, kChunks = T::kChunks;
    constexpr int kDepth = QT == 1 ? 3 : 2;                            // tiles in flight: what the registers hold (a third spills: prompt 331 us, not 303)
    constexpr int kSlot = QT * NB * 512 + 48 * QT;                     // floats of a partial result
    constexpr int kJoin = kKvJoin, kFinal = 8192;                         // parts added at a time; where the counters of the last sums begin
    __shared__ __align__(16) float comb[NW][kEl][4][64];
    __shared__ float ml[NW][QT][16][3];                                // maximum, sum, exact sum
    __shared__ int last;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, g = lane >> 4;
    KvItem it;
    if (!kv_find<NW * 32>(a, a.item0 + (int)blockIdx.x, kRows, QT == 1 ? 16 : 8, QT == 1 ? 3 : 4, &it))
        return;                                                        // (the whole workgroup)
    const int rows = it.n * a.group, row0 = it.tile * kRows;
    const int i0 = row0 / a.group, i1 = min((row0 + kRows - 1) / a.group, it.n - 1);
    const bool tree = a.tree != nullptr, causal = a.causal && !tree;
    const int hi = causal ? max(0, min(it.len, it.len - it.n + i1 + 1)) : it.len;
    const int lo = a.window > 0 ? max(0, it.len - it.n + i0 + 1 - a.window) & ~31 : 0;
    const int tiles = max(0, (hi - lo + 31) >> 5);
    const int t_begin = (lo >> 5) + part_begin(tiles, it.s, it.S), t_end = (lo >> 5) + part_begin(tiles, it.s + 1, it.S);
    // tiles from `plain_lo` on and up to `plain_hi` need no mask: every query of this workgroup sees all of their tokens
    const int plain_hi = causal ? it.len - it.n + i0 + 1 : tree ? it.len - it.n : it.len;
    const int plain_lo = a.window > 0 ? it.len - it.n + i1 + 1 - a.window : 0;

    bf16x8_t q[QT][NB];
    const KvSight sight = {it.len - it.n, a.window, causal, tree};
    int at_q[QT];                                                      // the positions of the lane's queries
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int row = row0 + qt * 16 + c;
        const int i = row / a.group, head = it.h * a.group + row - i * a.group;
        const bool live = row < rows;
        at_q[qt] = live ? it.len - it.n + i : kNobody;
        const uint16_t* from = a.q.p + (int64_t)(it.first + (live ? i : 0)) * a.q.token + (int64_t)(live ? head : it.h * a.group) * a.q.head;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            if (!kPad || 8 * NB * g + 8 * j < 32 * a.c.nb)
                q[qt][j] = *reinterpret_cast<const bf16x8_t*>(from + 8 * NB * g + 8 * j);
            else
                q[qt][j] = __builtin_bit_cast(bf16x8_t, (u32x4_t{0, 0, 0, 0}));
        }
    }

    f32x4_t o[QT][2 * NB];
    float m[QT], exact[QT];
    f32x4_t l[QT];
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        m[qt] = -INFINITY;
        l[qt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        exact[qt] = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * NB; ++e)
            o[qt][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    const float scale = a.scale;
    const bool wanted = a.lse != nullptr;                              // the logarithm of the sums
    auto compute = [&](T& t, int tile) {
        const int j0 = tile * 32;
        const bool whole = t.page[0] >= 0 && t.page[1] >= 0 && j0 + 32 <= it.len;
        const bool masked = !(whole && j0 + 32 <= plain_hi && j0 >= plain_lo);
        f32x4_t s[QT][2];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const bf16x8_t k = key_operand(t, h, j);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
                    s[qt][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[qt][j], j ? s[qt][h] : f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            }
        // Converts between the products, four for each operand: the matrix pipe works beside them in one wave's stream better than blocks of
        // either do in two waves' (9 new tokens each of 16 rows of 16000, dim 128: 168 us, 171 in the compiler's order; 5001 tokens of a prompt
        // 303 and 304; dim 64 within 1 %).
        __builtin_amdgcn_sched_group_barrier(0x2, 6, 0);
#pragma unroll
        for (int i = 0; i < 2 * NB * QT; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x2, 4 / QT, 0);
        }
        bool odd = false;                                              // the tile has values that may be no numbers
        if (masked) {
            uint64_t word[QT];
#pragma unroll
            for (int qt = 0; qt < QT; ++qt)
                word[qt] = sight.word(a, it, at_q[qt]);
            // Tokens behind the end and pages that are not there: whatever lies in the memory must not reach the sums.
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int here = t.page[h] < 0 ? 0 : it.len - j0 - 16 * h;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = j0 + 16 * h + 4 * g + i;
                    const bool there = 4 * g + i < here;
#pragma unroll
                    for (int qt = 0; qt < QT; ++qt)
                        s[qt][h][i] = there && sight.sees(at_q[qt], word[qt], j) ? s[qt][h][i] : -INFINITY;
#pragma unroll
                    for (int ch = 0; ch < kChunks; ++ch) {
                        if (!there)
                            clear_value(t, h, i, ch);
                        odd |= value_scale(t, h, i, ch) >= kOddScale;
                    }
                }
            }
            odd = __ballot(odd) != 0;
            if (odd)
                drop_odd_values(t);
        }
        bf16x8_t p[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            p[qt] = softmax_step<2 * NB>(s[qt], scale, wanted, &m[qt], &l[qt], &exact[qt], o[qt]);
        }
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
            bf16x8_t x[kEl];
            value_operands(t, ch, x);
#pragma unroll
            for (int e = 0; e < kEl; ++e)
#pragma unroll
                for (int qt = 0; qt < QT; ++qt)
                    o[qt][ch * kEl + e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[e], p[qt], o[qt][ch * kEl + e], 0, 0, 0);
        }
        if (odd) {
            // They are loaded once more (no register holds them over the product), for the queries that see them.
            load_tile(t, a.c, it.h, j0, t.page[0], t.page[1]);
            bf16x8_t seen[QT];
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                const uint64_t word = sight.word(a, it, at_q[qt]);
                u32x4_t y = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int j = j0 + 16 * (i >> 2) + 4 * g + (i & 3);
                    if (t.page[i >> 2] >= 0 && j < it.len && sight.sees(at_q[qt], word, j))
                        y[i >> 1] |= i & 1 ? 0x3F800000u : 0x3F80u;
                }
                seen[qt] = __builtin_bit_cast(bf16x8_t, y);
            }
#pragma unroll
            for (int ch = 0; ch < kChunks; ++ch)
                add_odd_values<QT, 2 * NB>(t, ch, seen, o);
        }
    };

    // Tiles t_begin + wave, + 4, ...: kDepth - 1 of them are on their way while one is used.
    int pages = 0, loaded = 0;
    auto load = [&](T& t, int tile) {
        if ((loaded & 31) == 0)
            pages = kv_pages32<NW>(a, it.b, it.len, tile);
        const int k = (loaded & 31) * 2;
        ++loaded;
        load_tile(t, a.c, it.h, tile * 32, __builtin_amdgcn_readlane(pages, k), __builtin_amdgcn_readlane(pages, k + 1));
    };
    int tile = t_begin + wave;
    if (tile < t_end) {
        T t[kDepth];
#pragma unroll
        for (int d = 0; d < kDepth - 1; ++d)
            if (tile + d * NW < t_end)
                load(t[d], tile + d * NW);
        for (bool more = true; more;) {
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                if (tile + (kDepth - 1) * NW < t_end)
                    load(t[(d + kDepth - 1) % kDepth], tile + (kDepth - 1) * NW);
                compute(t[d], tile);
                tile += NW;
                more = tile < t_end;
                if (!more)
                    break;
            }
        }
    }

    int64_t out_at[QT];                                                // where the lane's queries' results go, -1: no query
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const int row = row0 + qt * 16 + c, i = row / a.group;
        out_at[qt] = row < rows ? (int64_t)(it.first + i) * a.out.token + (int64_t)(it.h * a.group + row - i * a.group) * a.out.head : -1;
    }
    // The four waves' sums meet in the LDS, one chunk of elements at a time; wave i takes row i of the accumulators.
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const float sum = wanted ? sum_of_rows(exact[qt]) : 0.f;
        if (g == 0) {
            ml[wave][qt][c][0] = m[qt];
            ml[wave][qt][c][1] = l[qt][0];
            ml[wave][qt][c][2] = sum;
        }
    }
    float* part = a.part + (int64_t)(it.slot0 + it.s * it.slots) * kSlot;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        float f[NW], top = -INFINITY, total = 0.f, precise = 0.f;
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kEl; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    comb[wave][e][i][lane] = o[qt][ch * kEl + e][i];
            __syncthreads();
            if (ch == 0) {
#pragma unroll
                for (int w = 0; w < NW; ++w)
                    top = fmaxf(top, ml[w][qt][c][0]);
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    f[w] = ml[w][qt][c][0] == -INFINITY ? 0.f : exp2f((ml[w][qt][c][0] - top) * scale);
                    // (a wave that has met only NaN scores has no maximum, but its sum says so)
                    f[w] = ml[w][qt][c][1] != ml[w][qt][c][1] ? __uint_as_float(0x7FC00000u) : f[w];
                    total += f[w] * ml[w][qt][c][1];
                    precise += f[w] * ml[w][qt][c][2];
                }
            }
            float r[kEl];
#pragma unroll
            for (int e = 0; e < kEl; ++e) {
                r[e] = 0.f;
#pragma unroll
                for (int w = 0; w < NW; ++w)
                    r[e] += f[w] * comb[w][e][wave][lane];
            }
            if (it.S == 1) {
                if (out_at[qt] >= 0 && (!kPad || ch * T::kChunk + kEl * (4 * g + wave) < 32 * a.c.nb)) {
                    const float inv = total == 0.f ? 0.f : 1.f / total;
                    uint16_t* to = a.out.p + out_at[qt] + ch * T::kChunk + kEl * (4 * g + wave);
                    uint32_t y[kEl / 2];
#pragma unroll
                    for (int e = 0; e < kEl; e += 2)
                        y[e / 2] = f32_to_bf16_rne2(r[e] * inv, r[e + 1] * inv);
                    __builtin_memcpy(__builtin_assume_aligned(to, kEl * 2), y, kEl * 2);
                }
            } else {
#pragma unroll
                for (int e = 0; e < kEl; ++e)
                    put_through(&part[((qt * 2 * NB + ch * kEl + e) * 4 + wave) * 64 + lane], r[e]);
            }
        }
        if (wave == 0 && g == 0) {
            if (it.S > 1) {
                put_through(&part[QT * NB * 512 + qt * 48 + c], top);
                put_through(&part[QT * NB * 512 + qt * 48 + 16 + c], total);
                put_through(&part[QT * NB * 512 + qt * 48 + 32 + c], precise);
            } else if (a.lse && out_at[qt] >= 0) {
                const int row = row0 + qt * 16 + c, i = row / a.group;
                a.lse[(int64_t)(it.first + i) * (a.group * a.c.heads) + it.h * a.group + row - i * a.group] =
                    precise == 0.f ? -INFINITY : (top * scale + log2f(precise)) * kLn2;
            }
        }
    }
    if (it.S == 1)
        return;

    // Parts of one row of keys: of every kJoin parts the workgroup that comes last adds them, of these the one that comes last
    // again, in the order of the parts whoever it is.  Nobody waits.  The parts go past the L2 (each die has its own) with coherent stores,
    // which have arrived when the wave's counter of stores is at zero, so that the count needs no write-back of a whole L2 in front of
    // it: with __threadfence() in that place one row of 131071 tokens took 136 us, not 38.
    // Lanes without a query store and load as well, so that lines are whole and nothing branches (one token, 32 heads of their own, 2000
    // tokens: 10.4 us, 12.4 with those lanes left out).
    const float* parts = a.part + (int64_t)it.slot0 * kSlot;
    int first = it.s - it.s % kJoin, count = min(kJoin, it.S - first), step = 1;
    bool done = it.S <= kJoin;
    uint32_t* counter = &a.counters[it.slot0 + first * it.slots];
    while (true) {
        drain_vmem();
        __syncthreads();
        if (threadIdx.x == 0)
            last = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)count - 1;
        __syncthreads();
        if (!last)
            return;
        if (threadIdx.x == 0)
            __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const float* from = parts + (int64_t)first * it.slots * kSlot;
        const int64_t pitch = (int64_t)step * it.slots * kSlot;
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
            const bool live = out_at[qt] >= 0;
            float top = -INFINITY, total = 0.f, precise = 0.f;
            float r[2 * NB];
#pragma unroll
            for (int e = 0; e < 2 * NB; ++e)
                r[e] = 0.f;
            for (int s = 0; s < count; s += kJoin) {                   // (more than kJoin only for the last sum of very many parts)
                float ms[kJoin], ls[kJoin], es[kJoin], x[kJoin][2 * NB];
#pragma unroll
                for (int k = 0; k < kJoin; ++k) {
                    const float* p = from + min(s + k, count - 1) * pitch;
                    ms[k] = get_through(&p[QT * NB * 512 + qt * 48 + c]);
                    ls[k] = get_through(&p[QT * NB * 512 + qt * 48 + 16 + c]);
                    es[k] = get_through(&p[QT * NB * 512 + qt * 48 + 32 + c]);
#pragma unroll
                    for (int e = 0; e < 2 * NB; ++e)
                        x[k][e] = get_through(&p[((qt * 2 * NB + e) * 4 + wave) * 64 + lane]);
                }
                float now = top;
#pragma unroll
                for (int k = 0; k < kJoin; ++k)
                    now = fmaxf(now, ms[k]);
                const float old = top == -INFINITY ? 0.f : exp2f((top - now) * scale);
                total *= old;
                precise *= old;
#pragma unroll
                for (int e = 0; e < 2 * NB; ++e)
                    r[e] *= old;
                top = now;
#pragma unroll
                for (int k = 0; k < kJoin; ++k) {
                    float f = ms[k] == -INFINITY ? 0.f : exp2f((ms[k] - now) * scale);
                    f = ls[k] != ls[k] ? __uint_as_float(0x7FC00000u) : f;
                    f = s + k < count ? f : 0.f;
                    total += f * (s + k < count ? ls[k] : 0.f);
                    precise += f * (s + k < count ? es[k] : 0.f);
#pragma unroll
                    for (int e = 0; e < 2 * NB; ++e)
                        r[e] += s + k < count ? f * x[k][e] : 0.f;
                }
            }
            if (!done) {
                // In the place of the first of them, whose maximum and sums all four waves read and wave 0 replaces: no wave stores before
                // every wave's loads are here.  (`done` and the loops' bounds are the same for the whole workgroup.)
                drain_vmem();
                __syncthreads();
                float* to = const_cast<float*>(from);
#pragma unroll
                for (int e = 0; e < 2 * NB; ++e)
                    put_through(&to[((qt * 2 * NB + e) * 4 + wave) * 64 + lane], r[e]);
                if (wave == 0 && g == 0) {
                    put_through(&to[QT * NB * 512 + qt * 48 + c], top);
                    put_through(&to[QT * NB * 512 + qt * 48 + 16 + c], total);
                    put_through(&to[QT * NB * 512 + qt * 48 + 32 + c], precise);
                }
                continue;
            }
            if (!live)
                continue;
            const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
            for (int ch = 0; ch < kChunks; ++ch) {
                if (kPad && ch * T::kChunk + kEl * (4 * g + wave) >= 32 * a.c.nb)
                    continue;
                uint16_t* to = a.out.p + out_at[qt] + ch * T::kChunk + kEl * (4 * g + wave);
                uint32_t y[kEl / 2];
#pragma unroll
                for (int e = 0; e < kEl; e += 2)
                    y[e / 2] = f32_to_bf16_rne2(r[ch * kEl + e] * inv, r[ch * kEl + e + 1] * inv);
                __builtin_memcpy(__builtin_assume_aligned(to, kEl * 2), y, kEl * 2);
            }
            if (a.lse && wave == 0 && g == 0) {
                const int row = row0 + qt * 16 + c, i = row / a.group;
                a.lse[(int64_t)(it.first + i) * (a.group * a.c.heads) + it.h * a.group + row - i * a.group] =
                    precise == 0.f ? -INFINITY : (top * scale + log2f(precise)) * kLn2;
            }
        }
        if (done)
            return;
        count = (it.S + kJoin - 1) / kJoin;                            // and now the sums of the groups
        first = 0;
        step = kJoin;
        done = true;
        counter = &a.counters[kFinal + it.slot0];
    }
}

// Query tiles of a workgroup at most: two where an average sequence has more queries than one tile holds, and the registers hold the
// sums (8 times the tiles times dim / 32 of them).
static int most_query_tiles(int nb, int64_t queries) { return queries <= 16 || nb > 4 ? 1 : 2; }

// Two tiles decode a token once for both, one tile loads, combines and joins less in front of the first result: one where the
// workgroups with one tile run at once and all of them read less than 4096 tokens for each compute unit, as far as the table can
// tell the lengths: a table with room for more tokens than there are takes the rule past its border (us with one and with two: 4 new
// tokens, 64 heads on 8, over 1000: 9.6 and 13.1, 4 rows over 16000: 30.3 and 33.4, 16 rows over 4000: 30.1 and 28.0, over 16000: 94 and 76; prompts of
// 3000: 366 and 246, 5001: 454 and 303; dim 64, 9 tokens over 1000: 8.2 and 11.1, 16 rows of them over 16000: 49 and 42; dim 32 likewise 8.0 and 10.4,
// 68 and 72).  Heads of 96 elements run two tiles with 11 registers in scratch memory, and gain by it all the same: 16 rows over 16000 92 and
// 70, prompts of 3000 132 and 93.
static int query_tiles(const KvAttend& a, const DeviceInfo& dev)
{
    const int64_t queries = ((int64_t)a.b.tokens * a.group + a.b.rows - 1) / a.b.rows;
    if (most_query_tiles(a.c.nb, queries) == 1)
        return 1;
    const int64_t tiles = a.b.rows * ((queries + 15) / 16) * a.c.heads;
    int64_t tokens = (int64_t)a.b.width << a.c.shift;
    if (a.window > 0)
        tokens = std::min(tokens, a.window + queries / a.group);
    return tiles <= 2 * dev.cus && tiles * tokens < (int64_t)dev.cus * 4096 ? 1 : 2;
}

static int padded(int nb) { return nb == 3 ? 4 : nb == 6 ? 8 : nb; }

// Workgroups that the cutting aims for: two for each compute unit, as many as run at once up to dim 128. (Of dim 256 one runs at once: 8 rows
// of 16000 tokens, 16 heads on 2, take 29.1 us all the same, 35.6 with parts of twice the length; 32 rows of up to 8000 91 either way.)
static int attend_target(const DeviceInfo& dev) { return 2 * dev.cus; }

size_t kv_attend_part_bytes(int nb, int group, int64_t tokens, int64_t rows, const DeviceInfo& dev)
{
    const int qt = most_query_tiles(nb, rows ? (tokens * group + rows - 1) / rows : 0);
    return ((size_t)4 * attend_target(dev) + 8) * (qt * padded(nb) * 512 + 48 * qt) * sizeof(float);
}

template <int NB, bool kPad>
static hipError_t launch_attend(KvAttend a, int qt, int64_t blocks, hipStream_t stream)
{
    auto kernel = kv_attend_kernel<NB, 1, kPad>;
    if constexpr (NB <= 4)
        if (qt == 2)
            kernel = kv_attend_kernel<NB, 2, kPad>;
    // (Shares of one row may lie in two launches: nobody waits for a part, the last one joins.)
    for (int64_t i = 0; i < blocks; i += kKvMostBlocks) {
        a.item0 = (int)i;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(blocks - i, kKvMostBlocks)), dim3(256), 0, stream, a);
    }
    return hipGetLastError();
}

hipError_t launch_kv_attend(KvAttend a, const DeviceInfo& dev, hipStream_t stream)
{
    const int qt = query_tiles(a, dev);
    a.target = attend_target(dev);
    // No more workgroups than shares: 2 target + tiles x heads by the cutting, and no more than the tables' units.
    const int64_t per = 16 * qt;
    const int64_t tiles = a.b.starts ? (int64_t)a.b.tokens * a.group / per + a.b.rows : a.b.rows * (((int64_t)a.b.per_row * a.group + per - 1) / per);
    const int64_t units = (((int64_t)a.b.width << a.c.shift) + 127) / 128;
    int64_t blocks = tiles * a.c.heads + 2 * a.target;
    if (tiles * a.c.heads * units < blocks)
        blocks = tiles * a.c.heads * units;
    if (blocks > 0x7FFFFFFF)
        return hipErrorInvalidConfiguration;
    switch (a.c.nb) {
    case 1: return launch_attend<1, false>(a, qt, blocks, stream);
    case 2: return launch_attend<2, false>(a, qt, blocks, stream);
    case 3: return launch_attend<4, true>(a, qt, blocks, stream);
    case 4: return launch_attend<4, false>(a, qt, blocks, stream);
    case 6: return launch_attend<8, true>(a, qt, blocks, stream);
    case 8: return launch_attend<8, false>(a, qt, blocks, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace mxfp4
