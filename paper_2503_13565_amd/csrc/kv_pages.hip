// Who holds which page of a paged cache: forking, growing and cutting sequences on the device, so that a speculative step
// (drafts begun, tokens accepted or dropped) needs no word from the host and can be captured whole.  All integers; every
// result is the same on every run: a page's count is the sum of what was added and taken, free pages are taken from the lowest
// number on, by a scan.
#include "common.h"
#include "kv.h"

namespace mxfp4 {

__device__ __forceinline__ int pages_of(int tokens, int shift) { return (int)(((unsigned)tokens + (1u << shift) - 1) >> shift); }

// One workgroup per pair.  Several forks of one sequence add to the same counts (sums do not depend on their order).
__global__ __launch_bounds__(256) void kv_fork_kernel(KvPool p, const int32_t* src, const int32_t* dst)
{
    const int from = src[blockIdx.x], to = dst[blockIdx.x];
    if ((unsigned)from >= (unsigned)p.rows || (unsigned)to >= (unsigned)p.rows || from == to)
        return;
    const int n = max(p.lens[from], 0);
    const int held = min(pages_of(n, p.shift), p.width);
    for (int w = threadIdx.x; w < p.width; w += 256) {
        const int page = w < held ? p.table[(int64_t)from * p.ldt + w] : -1;
        p.table[(int64_t)to * p.ldt + w] = page;
        if ((unsigned)page < (unsigned)p.pages)
            atomicAdd(&p.refs[page], 1);
    }
    if (threadIdx.x == 0)
        p.lens[to] = n;
}

// One workgroup per sequence.  Whoever takes a page's last count sets its free bit; which thread that is does not matter.
__global__ __launch_bounds__(256) void kv_release_kernel(KvPool p, const int32_t* rows, const int32_t* keep)
{
    const int row = rows[blockIdx.x];
    if ((unsigned)row >= (unsigned)p.rows)
        return;
    const int old = max(p.lens[row], 0);
    const int now = min(old, max(keep[blockIdx.x], 0));
    __syncthreads();
    if (threadIdx.x == 0)
        p.lens[row] = now;
    const int last = min(pages_of(old, p.shift), p.width);
    for (int w = pages_of(now, p.shift) + threadIdx.x; w < last; w += 256) {
        int32_t* entry = &p.table[(int64_t)row * p.ldt + w];
        const int page = *entry;
        *entry = -1;
        if ((unsigned)page < (unsigned)p.pages && atomicSub(&p.refs[page], 1) == 1)
            atomicOr(&p.bits[page >> 5], 1u << (page & 31));
    }
}

// Inclusive sum over the workgroup's 1024 threads, in thread order; `sums` holds a number per wave.
__device__ __forceinline__ int block_scan(int v, int* sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int u = __shfl_up(v, d);
        v += lane >= d ? u : 0;
    }
    __syncthreads();                             // (the last scan's sums are read)
    if (lane == 63)
        sums[wave] = v;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < 16; ++w)
        before += w < wave ? sums[w] : 0;
    return v + before;
}

// One workgroup of 1024 threads: the rows are scanned for what each needs, the free bits for the pages of the lowest numbers.
// Free pages are dealt out 1024 words (32768 pages) at a time: their numbers go to a list in the LDS in order, then every
// page finds its row by bisection among the rows' sums.  Latency-bound: a chain of some twelve loads, scans and barriers.
__global__ __launch_bounds__(1024) void kv_extend_kernel(KvPool p, const int32_t* rows, const int32_t* add, int count, int32_t* copies,
                                                         int32_t* missing)
{
    extern __shared__ int lds[];
    int* sum = lds;                              // needs of rows 0 .. i together
    int* mine = sum + kKvMaxRows;                // the page that a row would leave, or -1
    int* first = mine + kKvMaxRows;              // where a row's first new page goes
    uint16_t* list = reinterpret_cast<uint16_t*>(first + kKvMaxRows);
    __shared__ int sums[16], bad, found;
    constexpr int kEach = kKvMaxRows / 1024;
    const int tid = threadIdx.x;
    if (tid == 0)
        bad = found = 0;
    int n[kEach], a[kEach], row[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = tid * kEach + j;
        row[j] = i < count ? rows[i] : -1;
        if ((unsigned)row[j] >= (unsigned)p.rows)
            row[j] = -1;
        n[j] = row[j] < 0 ? 0 : max(p.lens[row[j]], 0);
        a[j] = row[j] < 0 ? 0 : max(add[i], 0);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = tid * kEach + j;
        int page = -1;
        if ((int64_t)n[j] + a[j] > ((int64_t)p.width << p.shift)) {
            bad = 1;
            n[j] = a[j] = 0;
        } else if (a[j] > 0 && (n[j] & ((1 << p.shift) - 1))) {
            page = p.table[(int64_t)row[j] * p.ldt + (n[j] >> p.shift)];
            if ((unsigned)page >= (unsigned)p.pages || p.refs[page] < 2)
                page = -1;
        }
        mine[i] = page;
    }
    __syncthreads();
    int need[kEach], own = 0;
    bool copy[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = tid * kEach + j;
        copy[j] = false;
        if (mine[i] >= 0) {
            int before = 0;                      // rows in front of this one that leave the same page
            for (int k = 0; k < i; ++k)
                before += mine[k] == mine[i];
            copy[j] = p.refs[mine[i]] - before > 1;
        }
        const int w = pages_of(n[j], p.shift);
        need[j] = pages_of(n[j] + a[j], p.shift) - w + copy[j];
        first[i] = w - copy[j];
        own += need[j];
    }
    const int all = block_scan(own, sums);
    int at = all - own;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        at += need[j];
        sum[tid * kEach + j] = at;
        if (!copy[j])
            mine[tid * kEach + j] = -1;          // (everybody has counted: the scan above has barriers)
    }
    __syncthreads();
    const int total = sum[kKvMaxRows - 1];
    const int words = (p.pages + 31) >> 5;
    int have = 0;
    for (int w = tid; w < words; w += 1024)
        have += __popc(p.bits[w]);
    have = block_scan(have, sums);
    if (tid == 1023)
        found = have;
    __syncthreads();
    if (bad || found < total) {                  // the same for all: nothing is changed
        if (tid == 0)
            *missing = bad ? -1 : total - found;
        for (int i = tid; i < count; i += 1024)
            copies[2 * i] = copies[2 * i + 1] = -1;
        return;
    }
    if (tid == 0)
        *missing = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = tid * kEach + j;
        if (i < count) {
            if (!copy[j])
                copies[2 * i] = copies[2 * i + 1] = -1;
            if (row[j] >= 0)
                p.lens[row[j]] = n[j] + a[j];
        }
    }
    int done = 0;
    for (int w0 = 0; done < total; w0 += 1024) {
        const uint32_t word = w0 + tid < words ? p.bits[w0 + tid] : 0u;
        const int c = __popc(word);
        const int upto = block_scan(c, sums);
        if (tid == 1023)
            found = upto;
        const int left = total - done;           // of this tile's free pages, the first `left` are taken
        int k = upto - c;
        uint32_t rest = word;
        while (rest && k < left) {
            const int bit = __ffs(rest) - 1;
            rest &= rest - 1;
            list[k++] = (uint16_t)(tid * 32 + bit);
        }
        if (rest != word)
            p.bits[w0 + tid] = rest;
        __syncthreads();
        const int got = min(found, left);
        for (int r = tid; r < got; r += 1024) {
            const int rank = done + r, page = w0 * 32 + list[r];
            int lo = 0, hi = kKvMaxRows - 1;     // the first row whose sum passes the rank
            while (lo < hi) {
                const int m = (lo + hi) >> 1;
                if (sum[m] > rank)
                    hi = m;
                else
                    lo = m + 1;
            }
            const int k2 = rank - (lo ? sum[lo - 1] : 0);
            const int r2 = rows[lo];
            const int w = first[lo] + k2;
            p.refs[page] = 1;
            p.table[(int64_t)r2 * p.ldt + w] = page;
            if (k2 == 0 && mine[lo] >= 0) {      // the first one takes the place of the page that others hold too
                copies[2 * lo] = mine[lo];
                copies[2 * lo + 1] = page;
                atomicSub(&p.refs[mine[lo]], 1);
            }
        }
        __syncthreads();
        done += got;
    }
}

hipError_t launch_kv_fork(const KvPool& p, const int32_t* src, const int32_t* dst, int count, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_fork_kernel, dim3((unsigned)count), dim3(256), 0, stream, p, src, dst);
    return hipGetLastError();
}

hipError_t launch_kv_extend(const KvPool& p, const int32_t* rows, const int32_t* add, int count, int32_t* copies,
                            int32_t* missing, hipStream_t stream)
{
    constexpr int kBytes = 3 * kKvMaxRows * 4 + 1024 * 32 * 2;
    static LdsLimit limit;
    const hipError_t e = limit.raise(reinterpret_cast<const void*>(kv_extend_kernel), kBytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kv_extend_kernel, dim3(1), dim3(1024), kBytes, stream, p, rows, add, count, copies, missing);
    return hipGetLastError();
}

hipError_t launch_kv_release(const KvPool& p, const int32_t* rows, const int32_t* keep, int count, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_release_kernel, dim3((unsigned)count), dim3(256), 0, stream, p, rows, keep);
    return hipGetLastError();
}

}  // namespace mxfp4
