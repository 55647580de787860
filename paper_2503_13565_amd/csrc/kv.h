// Internal interface of the paged MXFP4 cache (include/mxfp4.h, mxfp4_kv_*): what the kernels get.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace mxfp4 {

constexpr int kKvMaxRows = 4096;             // sequences of one extend (its scans live in the LDS)
// Workgroups of 256 threads of one launch: the device counts a grid's threads along x in 32 bits, and what is past them is left out without
// an error.  Calls with more workgroups are several launches.
constexpr int kKvMostBlocks = 1 << 23;

// The cache: page p of array x at x + p * stride, [heads][page][dim / 2] or [heads][page][dim / 32] inside.
struct KvView {
    uint8_t* kq;
    uint8_t* ks;
    uint8_t* vq;
    uint8_t* vs;
    int64_t psq, pss;
    int pages, heads, shift, nb;             // shift: log2 of the tokens of a page; nb: dim / 32
};

// The batch: new tokens of row b are starts[b] .. starts[b + 1] - 1, or per_row each.
struct KvBatch {
    const int32_t* table;
    int64_t ldt;
    const int32_t* lens;
    const int32_t* starts;
    int rows, width, tokens, per_row;
    int t0;                                  // the launch's first token
};

struct KvTensor {
    uint16_t* p;
    int64_t token, head;
};

struct KvRope {
    const float* cos;
    const float* sin;
    const int32_t* positions;
    int length, dim;
};

struct KvAttend {
    KvView c;
    KvBatch b;
    KvTensor q, out;
    float* lse;
    const uint64_t* tree;
    int group, causal;                       // query heads per key/value head
    int window;                              // 0: none
    float scale;                             // times log2(e)
    int target;                              // workgroups that the cutting of long rows aims for
    int item0;                               // the launch's first share
    uint32_t* counters;
    float* part;
};

struct KvPool {
    int32_t* refs;
    uint32_t* bits;
    int32_t* table;
    int32_t* lens;
    int64_t ldt;
    int pages, shift, width, rows;
};

hipError_t launch_kv_append(const KvView& c, KvBatch b, const KvTensor& k, const KvTensor& v, const KvTensor& q,
                            const KvTensor& q_out, int q_heads, const KvRope& rope, hipStream_t stream);
hipError_t launch_kv_read(const KvView& c, KvBatch b, const KvTensor& k, const KvTensor& v, hipStream_t stream);
hipError_t launch_kv_compact(const KvView& c, const int32_t* table, int64_t ldt, int width, const int32_t* base,
                             const int32_t* keep, int ldk, const int32_t* counts, int rows, hipStream_t stream);
// `rows` (null: whole pages): only the slots in use before rows[i] grew by add[i] are copied (rounded up to 16).
hipError_t launch_kv_copy(const KvView& c, const int32_t* src, const int32_t* dst, int pitch, int count, const int32_t* rows,
                          int n_rows, const int32_t* lens, const int32_t* add, hipStream_t stream);

hipError_t launch_kv_fork(const KvPool& p, const int32_t* src, const int32_t* dst, int count, hipStream_t stream);
hipError_t launch_kv_extend(const KvPool& p, const int32_t* rows, const int32_t* add, int count, int32_t* copies,
                            int32_t* missing, hipStream_t stream);
hipError_t launch_kv_release(const KvPool& p, const int32_t* rows, const int32_t* keep, int count, hipStream_t stream);

// Attention: bytes of the partial results behind the counters, and the launch (kv_attend.hip).
size_t kv_attend_part_bytes(int nb, int group, int64_t tokens, int64_t rows, const DeviceInfo& dev);
hipError_t launch_kv_attend(KvAttend a, const DeviceInfo& dev, hipStream_t stream);

// Device side -----------------------------------------------------------------------------------------------------

// Row, position and number of new tokens of packed token t; starts are looked through by the whole wave, 64 at a time
// (t is the same in all lanes).  row < 0: no row has this token.
struct KvPlace {
    int row, at;
};
__device__ __forceinline__ KvPlace kv_place(const KvBatch& b, int t)
{
    KvPlace p;
    if (!b.starts) {
        p.row = t / b.per_row;
        p.at = b.lens[p.row] - b.per_row + (t - p.row * b.per_row);
        return p;
    }
    const int lane = threadIdx.x & 63;
    int at = -1;                             // how many starts are <= t, less one
    for (int base = 0; base <= b.rows; base += 64) {
        const int i = base + lane;
        const int s = i <= b.rows ? b.starts[i] : 0x7FFFFFFF;
        const int here = __popcll(__ballot(s <= t));
        at += here;
        if (here < 64)
            break;
    }
    if (at < 0 || at >= b.rows) {
        p.row = -1;
        p.at = -1;
        return p;
    }
    at = __builtin_amdgcn_readfirstlane(at);
    p.row = at;
    p.at = b.lens[at] - b.starts[at + 1] + t;
    return p;
}

// Inclusive sums over the wave's lanes, in the vector unit (through the LDS crossbar a step waits for its answer).
template <int kCtrl, int kRows>
__device__ __forceinline__ int dpp_or_zero(int v)
{
    return __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int v)
{
    v += dpp_or_zero<0x111, 0xF>(v);         // row_shr 1, 2, 4, 8: sums within 16 lanes
    v += dpp_or_zero<0x112, 0xF>(v);
    v += dpp_or_zero<0x114, 0xF>(v);
    v += dpp_or_zero<0x118, 0xF>(v);
    v += dpp_or_zero<0x142, 0xA>(v);         // the last lane of rows 0 and 2 to rows 1 and 3
    v += dpp_or_zero<0x143, 0xC>(v);         // lane 31 to the upper half
    return v;
}

// Page of position `at` of a row, or -1 where there is none.
__device__ __forceinline__ int kv_page(const int32_t* table, int64_t ldt, int width, int shift, int pages, int row, int at)
{
    if (row < 0 || at < 0 || (at >> shift) >= width)
        return -1;
    const int page = table[(int64_t)row * ldt + (at >> shift)];
    return (unsigned)page < (unsigned)pages ? page : -1;
}

}  // namespace mxfp4
