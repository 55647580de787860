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

// wave_scan for numbers below 2^31, whose sums stop there: rows may ask for 2^26 pages each, 2^38 together.
__device__ __forceinline__ int add_up_to_cap(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, 0x7FFFFFFFu); }
__device__ __forceinline__ int capped_wave_scan(int v)
{
    v = add_up_to_cap(v, dpp_or_zero<0x111, 0xF>(v));
    v = add_up_to_cap(v, dpp_or_zero<0x112, 0xF>(v));
    v = add_up_to_cap(v, dpp_or_zero<0x114, 0xF>(v));
    v = add_up_to_cap(v, dpp_or_zero<0x118, 0xF>(v));
    v = add_up_to_cap(v, dpp_or_zero<0x142, 0xA>(v));
    v = add_up_to_cap(v, dpp_or_zero<0x143, 0xC>(v));
    return v;
}

// Inclusive sums of two numbers over the workgroup's 1024 threads, in thread order, the sums of all, and that of a third number;
// `sums` holds three numbers per wave.  Those of `a` stop at 2^31 - 1.
struct Scan {
    int a, b, all_a, all_b, all_c;
};
__device__ __forceinline__ Scan block_scan(int a, int b, int c, int (*sums)[16])
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Scan s;
    s.a = capped_wave_scan(a);
    s.b = wave_scan(b);
    c = wave_scan(c);
    __syncthreads();                             // (the last scan's sums are read)
    if (lane == 63) {
        sums[0][wave] = s.a;
        sums[1][wave] = s.b;
        sums[2][wave] = c;
    }
    __syncthreads();
    const int upto_a = capped_wave_scan(lane < 16 ? sums[0][lane] : 0), upto_b = wave_scan(lane < 16 ? sums[1][lane] : 0);
    s.all_a = __builtin_amdgcn_readlane(upto_a, 15);
    s.all_b = __builtin_amdgcn_readlane(upto_b, 15);
    s.all_c = __builtin_amdgcn_readlane(wave_scan(lane < 16 ? sums[2][lane] : 0), 15);
    s.a = add_up_to_cap(s.a, wave ? __builtin_amdgcn_readlane(upto_a, max(wave - 1, 0)) : 0);
    s.b += wave ? __builtin_amdgcn_readlane(upto_b, max(wave - 1, 0)) : 0;
    return s;
}

// A word of the free bits; bits past the last page name no page, whatever they hold.
__device__ __forceinline__ uint32_t free_word(const KvPool& p, int words, int w)
{
    if (w >= words)
        return 0u;
    const int last = p.pages & 31;
    return p.bits[w] & (w == words - 1 && last ? (1u << last) - 1 : 0xFFFFFFFFu);
}

// One workgroup of 1024 threads: the rows are scanned for what each needs, the free bits for the pages of the lowest numbers.
// Free pages are dealt out 1024 words (32768 pages) at a time: their numbers go to a list in the LDS in order, then every
// page finds its row by bisection among the rows' sums.  Latency-bound: a chain of some ten loads, scans and barriers.
// kEach: rows of a thread, 1 up to 1024 rows (8 rows: 4.7 us, 7.7 with four), 4 up to 4096.
template <int kEach>
__global__ __launch_bounds__(1024) void kv_extend_kernel(KvPool p, const int32_t* rows, const int32_t* add, int count, int32_t* copies,
                                                         int32_t* missing)
{
    extern __shared__ __align__(16) int lds[];
    constexpr int kRows = 1024 * kEach;
    int* mine = lds;                             // the page that a row would leave, or -1
    int* sum = mine + kRows;                     // needs of rows 0 .. i together
    int* first = sum + kRows;                    // where a row's first new page goes
    uint16_t* list = reinterpret_cast<uint16_t*>(first + kRows);
    __shared__ int sums[3][16], bad;
    const int tid = threadIdx.x;
    if (tid == 0)
        bad = 0;
    const int words = (p.pages + 31) >> 5;
    const uint32_t word0 = free_word(p, words, tid);                   // (asked for before the rows' chain of loads)
    int n[kEach], a[kEach], row[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = tid * kEach + j;
        row[j] = i < count ? rows[i] : -1;
        a[j] = i < count ? max(add[i], 0) : 0;
        if ((unsigned)row[j] >= (unsigned)p.rows)
            row[j] = -1;
        n[j] = row[j] < 0 ? 0 : max(p.lens[row[j]], 0);
        a[j] = row[j] < 0 ? 0 : a[j];
    }
    int more = 0;                                // free pages of the words behind
    for (int w = 1024 + tid; w < words; w += 1024)
        more += __popc(free_word(p, words, w));
    __syncthreads();
    int refs[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        int page = -1;
        refs[j] = 0;
        if ((int64_t)n[j] + a[j] > ((int64_t)p.width << p.shift)) {
            bad = 1;
            n[j] = a[j] = 0;
        } else if (a[j] > 0 && (n[j] & ((1 << p.shift) - 1))) {
            page = p.table[(int64_t)row[j] * p.ldt + (n[j] >> p.shift)];
            if ((unsigned)page < (unsigned)p.pages)
                refs[j] = p.refs[page];
            if (refs[j] < 2)
                page = -1;
        }
        mine[tid * kEach + j] = page;
    }
    __syncthreads();                             // (everybody sees `mine`)
    int need[kEach], own = 0;
    bool copy[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = tid * kEach + j, page = mine[i];
        copy[j] = false;
        if (page >= 0) {
            int before = 0;                      // rows in front of this one that leave the same page
            const int4* at = reinterpret_cast<const int4*>(mine);
            for (int k = 0; k < i >> 2; ++k)
                before += (at[k].x == page) + (at[k].y == page) + (at[k].z == page) + (at[k].w == page);
            for (int k = i & ~3; k < i; ++k)
                before += mine[k] == page;
            copy[j] = refs[j] - before > 1;
        }
        const int w = pages_of(n[j], p.shift);
        need[j] = pages_of(n[j] + a[j], p.shift) - w + copy[j];
        first[i] = w - copy[j];
        own += need[j];
    }
    Scan scan = block_scan(own, __popc(word0), more, sums);
    // (a total at the cap is past every number of pages; below it no sum has stopped)
    const int total = scan.all_a, free_pages = scan.all_b + scan.all_c;
    int at = scan.a - own;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = tid * kEach + j;
        at += need[j];
        sum[i] = at;
        if (!copy[j])
            mine[i] = -1;                        // (everybody has counted: the scan above has barriers)
    }
    if (bad || free_pages < total) {             // the same for all: nothing is changed
        if (tid == 0)
            *missing = bad ? -1 : total - free_pages;
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
        const uint32_t word = w0 == 0 ? word0 : free_word(p, words, w0 + tid);
        if (w0)
            scan = block_scan(0, __popc(word), 0, sums);
        const int found = scan.all_b, left = total - done;             // of this tile's free pages, the first `left` are taken
        int k = scan.b - __popc(word);
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
            int lo = 0, hi = count - 1;          // the first row whose sum passes the rank
            while (lo < hi) {
                const int m = (lo + hi) >> 1;
                if (sum[m] > rank)
                    hi = m;
                else
                    lo = m + 1;
            }
            const int k2 = rank - (lo ? sum[lo - 1] : 0);
            const int w = first[lo] + k2;
            p.refs[page] = 1;
            p.table[(int64_t)rows[lo] * p.ldt + w] = page;
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
    const bool few = count <= 1024;
    auto kernel = few ? kv_extend_kernel<1> : kv_extend_kernel<4>;
    const int bytes = 3 * 4 * (few ? 1024 : kKvMaxRows) + 1024 * 32 * 2;
    static LdsLimit limit[2];
    const hipError_t e = limit[few].raise(reinterpret_cast<const void*>(kernel), bytes);
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(kernel, dim3(1), dim3(1024), bytes, stream, p, rows, add, count, copies, missing);
    return hipGetLastError();
}

hipError_t launch_kv_release(const KvPool& p, const int32_t* rows, const int32_t* keep, int count, hipStream_t stream)
{
    hipLaunchKernelGGL(kv_release_kernel, dim3((unsigned)count), dim3(256), 0, stream, p, rows, keep);
    return hipGetLastError();
}

}  // namespace mxfp4
