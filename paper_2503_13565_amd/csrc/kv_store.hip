// Into, out of and inside a paged MXFP4 cache for gfx950: the store of new tokens (rotary positions and the cast of
// arXiv 2503.13565, section 3.4.3, in one launch), the values back out, tokens moved together, pages copied.
#include <algorithm>

#include "cast_block.h"
#include "common.h"
#include "kv.h"

namespace mxfp4 {

// Eight pairs of elements turned by eight angles: (x, y) -> (x cos - y sin, y cos + x sin).  Each product is rounded to FP32 on its
// own (no fused multiply-add), so that the BF16 result does not depend on how a compiler contracts.  kFirst, kSecond: which
// of the two is wanted.
template <bool kFirst, bool kSecond>
__device__ __forceinline__ void turn8(u32x4_t* x, u32x4_t* y, const KvRope& rope, int pos, int i)
{
#pragma clang fp contract(off)
    const bool inside = (unsigned)pos < (unsigned)rope.length;
    const int64_t at = (int64_t)(inside ? pos : 0) * (rope.dim >> 1) + i;
    f32x4_t c[2], s[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        c[j] = *reinterpret_cast<const f32x4_t*>(rope.cos + at + 4 * j);
        s[j] = *reinterpret_cast<const f32x4_t*>(rope.sin + at + 4 * j);
    }
    const float wrong = __uint_as_float(0x7FC00000u);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float r[2], t[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float u = bf16_bits_to_f32(k ? (*x)[j] >> 16 : (*x)[j] & 0xFFFFu);
            const float v = bf16_bits_to_f32(k ? (*y)[j] >> 16 : (*y)[j] & 0xFFFFu);
            const float co = c[(2 * j + k) >> 2][(2 * j + k) & 3], si = s[(2 * j + k) >> 2][(2 * j + k) & 3];
            const float uc = u * co, vs = v * si, vc = v * co, us = u * si;
            r[k] = inside ? uc - vs : wrong;
            t[k] = inside ? vc + us : wrong;
        }
        if (kFirst)
            (*x)[j] = f32_to_bf16_rne2(r[0], r[1]);
        if (kSecond)
            (*y)[j] = f32_to_bf16_rne2(t[0], t[1]);
    }
}

// A token's place in the cache, for one head.
struct KvSlot {
    uint8_t* q;
    uint8_t* s;
};
__device__ __forceinline__ KvSlot kv_slot(const KvView& c, bool keys, int page, int head, int at)
{
    const int64_t slot = (head << c.shift) + (at & ((1 << c.shift) - 1));
    return {(keys ? c.kq : c.vq) + (int64_t)page * c.psq + slot * (c.nb * 16), (keys ? c.ks : c.vs) + (int64_t)page * c.pss + slot * c.nb};
}

// Eight elements cast and stored; a quad of lanes has one block.  (All four take part, also without a page.)
__device__ __forceinline__ void kv_put(const u32x4_t x, const KvSlot& to, bool there, int e)
{
    uint32_t packed;
    int scale;
    cast_group<true>(x, &packed, &scale);
    if (!there)
        return;
    *reinterpret_cast<uint32_t*>(to.q + (e >> 1)) = packed;
    if ((e & 31) == 0)
        to.s[e >> 5] = (uint8_t)scale;
}

// Heads whose elements i and i + dim / 2 are turned together (or not at all), with whole blocks in either half: a thread takes
// eight of each half of a head of q, then of k, then of v, so that the angles are loaded once and every element once.
// Bound by latency for a step's few tokens (the token's row, its length and its page are one load behind the other, the
// elements are asked for in front of them) and by HBM for prompts.
__global__ __launch_bounds__(256) void kv_append_halves_kernel(KvView c, KvBatch b, KvTensor k, KvTensor v, KvTensor q, KvTensor qo,
                                                               int q_heads, KvRope rope)
{
    const int t = b.t0 + (int)blockIdx.x, g = blockIdx.y * 256 + threadIdx.x;
    const int half = c.nb * 2;                                         // groups of eight in half a head; a multiple of four
    const int head_all = (int)((unsigned)g / (unsigned)half), e = (g - head_all * half) * 8, e2 = e + half * 8;
    const bool live = head_all < q_heads + 2 * c.heads;                // the same for a whole quad
    const int what = head_all < q_heads ? 0 : head_all < q_heads + c.heads ? 1 : 2;
    const int head = what == 0 ? head_all : what == 1 ? head_all - q_heads : head_all - q_heads - c.heads;
    const KvTensor& in = what == 0 ? q : what == 1 ? k : v;
    const uint16_t* row = in.p + (int64_t)t * in.token + (int64_t)head * in.head;
    u32x4_t x = {0, 0, 0, 0}, y = {0, 0, 0, 0};
    if (live) {
        x = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row + e));
        y = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(row + e2));
    }
    const KvPlace at = kv_place(b, t);                                 // (with all lanes of the wave)
    if (!live)
        return;
    if (what < 2 && rope.dim)
        turn8<true, true>(&x, &y, rope, rope.positions ? rope.positions[t] : at.at, e);
    if (what == 0) {
        uint16_t* to = qo.p + (int64_t)t * qo.token + (int64_t)head * qo.head;
        *reinterpret_cast<u32x4_t*>(to + e) = x;                       // (the attention behind this call reads them)
        *reinterpret_cast<u32x4_t*>(to + e2) = y;
        return;
    }
    const int page = kv_page(b.table, b.ldt, b.width, c.shift, c.pages, at.row, at.at);
    const KvSlot to = kv_slot(c, what == 1, max(page, 0), head, at.at);
    kv_put(x, to, page >= 0, e);
    kv_put(y, to, page >= 0, e2);
}

// Any head and any rotary dim: 256 groups of eight elements of one token, the partner of a turned element by another load, and a pair's
// angles by both of its threads.  That is what bounds it for prompts: 9300 tokens of 32 + 64 heads of 128 of which 64 or 32 elements are turned
// take 120 us for 347 MB (the halves of whole heads 78 for 350), heads of 96 87 us for 262 MB.  A step's 108 tokens take 4.3 us, 3.9 in halves.
__global__ __launch_bounds__(256) void kv_append_kernel(KvView c, KvBatch b, KvTensor k, KvTensor v, KvTensor q, KvTensor qo,
                                                        int q_heads, KvRope rope)
{
    const int t = b.t0 + (int)blockIdx.x, g = blockIdx.y * 256 + threadIdx.x;
    const int per_head = c.nb * 4;
    const int head_all = g / per_head, e = (g - head_all * per_head) * 8;
    const bool live = head_all < q_heads + 2 * c.heads;                // the same for a whole quad (per_head is a multiple of four)
    const int what = head_all < q_heads ? 0 : head_all < q_heads + c.heads ? 1 : 2;
    const int head = what == 0 ? head_all : what == 1 ? head_all - q_heads : head_all - q_heads - c.heads;
    const KvTensor& in = what == 0 ? q : what == 1 ? k : v;
    const uint16_t* row = in.p + (int64_t)t * in.token + (int64_t)head * in.head;
    u32x4_t x = {0, 0, 0, 0};
    if (live)
        x = *reinterpret_cast<const u32x4_t*>(row + e);
    const KvPlace at = kv_place(b, t);                                 // (with all lanes of the wave)
    if (!live)
        return;
    if (what < 2 && e < rope.dim) {
        const int half = rope.dim >> 1, pos = rope.positions ? rope.positions[t] : at.at;
        u32x4_t other = *reinterpret_cast<const u32x4_t*>(row + (e < half ? e + half : e - half));
        if (e < half)
            turn8<true, false>(&x, &other, rope, pos, e);
        else
            turn8<false, true>(&other, &x, rope, pos, e - half);
    }
    if (what == 0) {
        *reinterpret_cast<u32x4_t*>(qo.p + (int64_t)t * qo.token + (int64_t)head * qo.head + e) = x;
        return;
    }
    const int page = kv_page(b.table, b.ldt, b.width, c.shift, c.pages, at.row, at.at);
    kv_put(x, kv_slot(c, what == 1, max(page, 0), head, at.at), page >= 0, e);
}

// Codes back to BF16 (exact: a code times a power of two), zeros where the token is nowhere.  Bound by the writes, four bytes
// for one that is read; they are not read again soon and go past the L2's order of use.
__global__ __launch_bounds__(256) void kv_read_kernel(KvView c, KvBatch b, KvTensor k, KvTensor v)
{
    const int t = b.t0 + (int)blockIdx.x, g = blockIdx.y * 256 + threadIdx.x;
    const int per_head = c.nb * 4;                                     // groups of eight elements
    const int head_all = (int)((unsigned)g / (unsigned)per_head), e = (g - head_all * per_head) * 8;
    const KvPlace at = kv_place(b, t);                                 // (with all lanes of the wave)
    const int page = kv_page(b.table, b.ldt, b.width, c.shift, c.pages, at.row, at.at);
    if (head_all >= 2 * c.heads)
        return;
    const bool keys = head_all < c.heads;
    const int head = keys ? head_all : head_all - c.heads;
    const KvTensor& out = keys ? k : v;
    if (!out.p)
        return;
    u32x4_t x = {0, 0, 0, 0};
    if (page >= 0) {
        const KvSlot from = kv_slot(c, keys, page, head, at.at);
        const uint32_t w = *reinterpret_cast<const uint32_t*>(from.q + (e >> 1));
        const float s = __uint_as_float((uint32_t)from.s[e >> 5] << 23);
        x[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
        x[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
        x[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
        x[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
    }
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4_t*>(out.p + (int64_t)t * out.token + (int64_t)head * out.head + e));
}

// Tokens of one sequence and one head move together, in place.  256 threads hold 256 / (2 nb) tokens at a time, one block (16
// bytes of codes and a scale byte) of a key or value each; a step's tokens are all read before any is written.  Bound by latency: the count,
// the kept place, the two pages and the token are loads one behind the other (48 trees' accepted tokens, 64 heads: 6.5 us, 1.1 for their
// bytes).  A step writes below
// what later steps read (keep ascends, so token j comes from beyond position j), so the steps need no more than that.
__global__ __launch_bounds__(256) void kv_compact_kernel(KvView c, const int32_t* table, int64_t ldt, int width, const int32_t* base,
                                                         const int32_t* keep, int ldk, const int32_t* counts)
{
    const int row = blockIdx.x, head = blockIdx.y;
    const int each = 2 * c.nb, at_once = 256 / each;
    const int tok = threadIdx.x / each, unit = threadIdx.x - tok * each;
    const bool keys = unit < c.nb;
    const int block = keys ? unit : unit - c.nb;
    const int n = min(counts[row], ldk), from0 = base[row];
    uint8_t* cq = keys ? c.kq : c.vq;
    uint8_t* cs = keys ? c.ks : c.vs;
    const int mask = (1 << c.shift) - 1;
    for (int i0 = 0; i0 < n; i0 += at_once) {
        const int i = i0 + tok;
        u32x4_t w = {0, 0, 0, 0};
        uint8_t s = 0;
        int to = -1, slot = 0;
        if (tok < at_once && i < n) {
            const int k = keep[(int64_t)row * ldk + i];
            if (k > i && from0 >= 0 && k <= 0x7FFFFFFF - from0) {
                const int from = kv_page(table, ldt, width, c.shift, c.pages, row, from0 + k);
                to = from < 0 ? -1 : kv_page(table, ldt, width, c.shift, c.pages, row, from0 + i);
                const int at = (head << c.shift) + ((from0 + k) & mask);
                slot = (head << c.shift) + ((from0 + i) & mask);
                if (to >= 0) {
                    w = *reinterpret_cast<const u32x4_t*>(cq + (int64_t)from * c.psq + ((int64_t)at * c.nb + block) * 16);
                    s = cs[(int64_t)from * c.pss + (int64_t)at * c.nb + block];
                }
            }
        }
        drain_vmem();                            // what this step reads is here before anyone writes
        __syncthreads();
        if (to >= 0) {
            *reinterpret_cast<u32x4_t*>(cq + (int64_t)to * c.psq + ((int64_t)slot * c.nb + block) * 16) = w;
            cs[(int64_t)to * c.pss + (int64_t)slot * c.nb + block] = s;
        }
    }
}

// Pages (or the slots of them that are in use) copied, one pair per blockIdx.x, 16 bytes at a time; a head's part of a page is
// a run of its own.
__global__ __launch_bounds__(256) void kv_copy_kernel(KvView c, const int32_t* src, const int32_t* dst, int pitch, const int32_t* rows,
                                                      int n_rows, const int32_t* lens, const int32_t* add)
{
    const int from = src[(int64_t)blockIdx.x * pitch], to = dst[(int64_t)blockIdx.x * pitch];
    const int row = rows ? rows[blockIdx.x] : 0, grown = rows ? add[blockIdx.x] : 0;   // (asked for with the pages)
    if ((unsigned)from >= (unsigned)c.pages || (unsigned)to >= (unsigned)c.pages || (rows && (unsigned)row >= (unsigned)n_rows))
        return;
    int tokens = 1 << c.shift;
    if (rows)
        tokens = (((lens[row] - grown) & (tokens - 1)) + 15) & ~15;
    const int q_run = tokens * c.nb, s_run = tokens * c.nb / 16;         // 16-byte pieces of a head
    const int q_page = c.nb << c.shift, s_page = (c.nb << c.shift) / 16;
    const int each = 2 * (q_run + s_run), total = each * c.heads;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < total; i += gridDim.y * 256) {
        const int head = i / each;
        int at = i - head * each;
        const bool keys = at < q_run + s_run;
        at = keys ? at : at - q_run - s_run;
        const bool codes = at < q_run;
        uint8_t* x = codes ? (keys ? c.kq : c.vq) : (keys ? c.ks : c.vs);
        const int64_t stride = codes ? c.psq : c.pss;
        const int64_t off = 16 * (codes ? (int64_t)head * q_page + at : (int64_t)head * s_page + at - q_run);
        *reinterpret_cast<u32x4_t*>(x + (int64_t)to * stride + off) = *reinterpret_cast<const u32x4_t*>(x + (int64_t)from * stride + off);
    }
}

hipError_t launch_kv_append(const KvView& c, KvBatch b, const KvTensor& k, const KvTensor& v, const KvTensor& q,
                            const KvTensor& qo, int q_heads, const KvRope& rope, hipStream_t stream)
{
    const bool halves = c.nb % 2 == 0 && (rope.dim == 0 || rope.dim == c.nb * 32);
    const int64_t groups = (int64_t)(q_heads + 2 * c.heads) * c.nb * (halves ? 2 : 4);
    for (; b.t0 < b.tokens; b.t0 += kKvMostBlocks)
        hipLaunchKernelGGL(halves ? kv_append_halves_kernel : kv_append_kernel,
                           dim3((unsigned)std::min(b.tokens - b.t0, kKvMostBlocks), (unsigned)((groups + 255) / 256)), dim3(256), 0, stream, c, b, k,
                           v, q, qo, q_heads, rope);
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvView& c, KvBatch b, const KvTensor& k, const KvTensor& v, hipStream_t stream)
{
    const int64_t groups = (int64_t)2 * c.heads * c.nb * 4;
    for (; b.t0 < b.tokens; b.t0 += kKvMostBlocks)
        hipLaunchKernelGGL(kv_read_kernel, dim3((unsigned)std::min(b.tokens - b.t0, kKvMostBlocks), (unsigned)((groups + 255) / 256)), dim3(256), 0,
                           stream, c, b, k, v);
    return hipGetLastError();
}

hipError_t launch_kv_compact(const KvView& c, const int32_t* table, int64_t ldt, int width, const int32_t* base,
                             const int32_t* keep, int ldk, const int32_t* counts, int rows, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_compact_kernel, dim3((unsigned)rows, (unsigned)c.heads), dim3(256), 0, stream, c, table, ldt, width, base, keep,
                       ldk, counts);
    return hipGetLastError();
}

hipError_t launch_kv_copy(const KvView& c, const int32_t* src, const int32_t* dst, int pitch, int count, const int32_t* rows,
                          int n_rows, const int32_t* lens, const int32_t* add, hipStream_t stream)
{
    const int64_t pieces = (int64_t)2 * c.heads * ((c.nb << c.shift) + (c.nb << c.shift) / 16);
    // A piece for each thread while that is about a thousand workgroups: eight begun pages of 32 heads then take 3.1 us, not 4.0 with four
    // pieces each; more workgroups only add to the calls in which few rows have a page to copy.
    int64_t blocks = (pieces + 255) / 256;
    const int64_t most = 1024 / count + 1;
    blocks = blocks < most ? blocks : most;
    for (int64_t i = 0; i < count; i += kKvMostBlocks)              // (`rows` come with at most kKvMaxRows pairs)
        hipLaunchKernelGGL(kv_copy_kernel, dim3((unsigned)std::min<int64_t>(count - i, kKvMostBlocks), (unsigned)blocks), dim3(256), 0, stream, c,
                           src + i * pitch, dst + i * pitch, pitch, rows, n_rows, lens, add);
    return hipGetLastError();
}

}  // namespace mxfp4
