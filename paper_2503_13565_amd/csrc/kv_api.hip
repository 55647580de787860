// C ABI of the paged MXFP4 cache (include/mxfp4.h, mxfp4_kv_*): argument checks and launches.  As everywhere in the library, the
// work goes to the caller's stream, and nothing here synchronises, allocates or frees device memory.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "kv.h"
#include "../../include/mxfp4.h"

namespace mxfp4 {

static bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

static int page_shift(int64_t page)
{
    for (int s = 4; s <= 10; ++s)
        if (page == (int64_t)1 << s)
            return s;
    return -1;
}

static int check_cache(const mxfp4_kv_cache* c, KvView* out)
{
    if (!c || !c->kq || !c->ks || !c->vq || !c->vs)
        return fail(MXFP4_ERR_NULL, "the cache or one of its arrays is NULL");
    const int shift = page_shift(c->page);
    if (shift < 0)
        return fail(MXFP4_ERR_SHAPE, "page=%d must be a power of two in [16, 1024]", c->page);
    const int d = c->dim;
    if (d != 32 && d != 64 && d != 96 && d != 128 && d != 192 && d != 256)
        return fail(MXFP4_ERR_SHAPE, "dim=%d must be 32, 64, 96, 128, 192 or 256", d);
    if (c->heads < 1 || c->heads > 65535)
        return fail(MXFP4_ERR_SHAPE, "heads=%d out of range [1, 65535]", c->heads);
    if (c->pages < 1 || c->pages > 0x7FFFFFFF)
        return fail(MXFP4_ERR_SHAPE, "pages=%lld out of range", (long long)c->pages);
    const int64_t least = (int64_t)c->heads * c->page * (d / 32);
    if (c->page_stride_q < least * 16 || c->page_stride_s < least)
        return fail(MXFP4_ERR_SHAPE, "page strides %lld, %lld are less than a page (%lld, %lld bytes)", (long long)c->page_stride_q,
                    (long long)c->page_stride_s, (long long)(least * 16), (long long)least);
    if (!aligned(c->kq, 16) || !aligned(c->ks, 16) || !aligned(c->vq, 16) || !aligned(c->vs, 16) || c->page_stride_q % 16 ||
        c->page_stride_s % 16)
        return fail(MXFP4_ERR_ALIGN, "the cache's arrays and page strides must be 16-byte aligned");
    out->kq = static_cast<uint8_t*>(c->kq);
    out->ks = static_cast<uint8_t*>(c->ks);
    out->vq = static_cast<uint8_t*>(c->vq);
    out->vs = static_cast<uint8_t*>(c->vs);
    out->psq = c->page_stride_q;
    out->pss = c->page_stride_s;
    out->pages = (int)c->pages;
    out->heads = c->heads;
    out->shift = shift;
    out->nb = d / 32;
    return MXFP4_OK;
}

static int check_table(const void* table, int64_t ldt, int64_t width, int shift)
{
    if (!table)
        return fail(MXFP4_ERR_NULL, "table is NULL");
    if (width < 1 || (width << shift) > 0x40000000 || ldt < width)
        return fail(MXFP4_ERR_SHAPE, "width=%lld (ldt=%lld): at least 1, ldt at least width, at most 2^30 tokens in a row", (long long)width,
                    (long long)ldt);
    if (!aligned(table, 4))
        return fail(MXFP4_ERR_ALIGN, "table must be 4-byte aligned");
    return MXFP4_OK;
}

static int check_batch(const mxfp4_kv_rows* b, int shift, KvBatch* out)
{
    if (!b)
        return fail(MXFP4_ERR_NULL, "the batch is NULL");
    if (b->tokens < 0 || b->tokens > 0x3FFFFFFF || b->rows < 0 || b->rows > (1 << 20))
        return fail(MXFP4_ERR_SHAPE, "rows=%lld or tokens=%lld out of range", (long long)b->rows, (long long)b->tokens);
    if (b->tokens == 0)
        return MXFP4_OK;
    if (b->rows == 0)
        return fail(MXFP4_ERR_SHAPE, "%lld tokens of no row", (long long)b->tokens);
    if (!b->lens)
        return fail(MXFP4_ERR_NULL, "lens is NULL");
    const int rc = check_table(b->table, b->ldt, b->width, shift);
    if (rc)
        return rc;
    if (!b->starts && b->tokens % b->rows)
        return fail(MXFP4_ERR_SHAPE, "without starts, tokens=%lld must be a multiple of rows=%lld", (long long)b->tokens, (long long)b->rows);
    if (!aligned(b->lens, 4) || !aligned(b->starts, 4))
        return fail(MXFP4_ERR_ALIGN, "lens and starts must be 4-byte aligned");
    out->table = b->table;
    out->ldt = b->ldt;
    out->lens = b->lens;
    out->starts = b->starts;
    out->rows = (int)b->rows;
    out->width = (int)b->width;
    out->tokens = (int)b->tokens;
    out->per_row = b->starts ? 0 : (int)(b->tokens / b->rows);
    return MXFP4_OK;
}

static int check_tensor(const mxfp4_kv_tensor* t, const char* what, KvTensor* out)
{
    if (!t || !t->data)
        return fail(MXFP4_ERR_NULL, "%s is NULL", what);
    if (t->token < 0 || t->head < 0)
        return fail(MXFP4_ERR_SHAPE, "%s: strides %lld, %lld are negative", what, (long long)t->token, (long long)t->head);
    if (!aligned(t->data, 16) || t->token % 8 || t->head % 8)
        return fail(MXFP4_ERR_ALIGN, "%s must be 16-byte aligned with strides that are multiples of 8", what);
    out->p = static_cast<uint16_t*>(t->data);
    out->token = t->token;
    out->head = t->head;
    return MXFP4_OK;
}

static int check_pool(const mxfp4_kv_pool* p, int64_t count, KvPool* out)
{
    if (!p)
        return fail(MXFP4_ERR_NULL, "the pool is NULL");
    if (count < 0 || count > (1 << 20))
        return fail(MXFP4_ERR_SHAPE, "count=%lld out of range", (long long)count);
    if (!p->refs || !p->free_bits || !p->lens)
        return fail(MXFP4_ERR_NULL, "refs, free_bits or lens is NULL");
    const int shift = page_shift(p->page);
    if (shift < 0)
        return fail(MXFP4_ERR_SHAPE, "page=%lld must be a power of two in [16, 1024]", (long long)p->page);
    if (p->pages < 1 || p->pages > 0x7FFFFFFF - 32768 || p->rows < 1 || p->rows > 0x7FFFFFFF)
        return fail(MXFP4_ERR_SHAPE, "pages=%lld or rows=%lld out of range", (long long)p->pages, (long long)p->rows);
    const int rc = check_table(p->table, p->ldt, p->width, shift);
    if (rc)
        return rc;
    if (!aligned(p->refs, 4) || !aligned(p->free_bits, 4) || !aligned(p->lens, 4))
        return fail(MXFP4_ERR_ALIGN, "refs, free_bits and lens must be 4-byte aligned");
    out->refs = p->refs;
    out->bits = p->free_bits;
    out->table = p->table;
    out->lens = p->lens;
    out->ldt = p->ldt;
    out->pages = (int)p->pages;
    out->shift = shift;
    out->width = (int)p->width;
    out->rows = (int)p->rows;
    return MXFP4_OK;
}

static int launched(hipError_t e, const char* what) { return e == hipSuccess ? MXFP4_OK : hip_fail(e, what); }

}  // namespace mxfp4

using namespace mxfp4;

extern "C" {

int mxfp4_kv_append(const mxfp4_kv_cache* cache, const mxfp4_kv_rows* batch, const mxfp4_kv_tensor* k,
                    const mxfp4_kv_tensor* v, const mxfp4_kv_tensor* q, const mxfp4_kv_tensor* q_out, int64_t q_heads,
                    const mxfp4_kv_rope* rope, void* stream)
{
    begin_call();
    KvView c;
    KvBatch b = {};
    KvTensor kt, vt, qt = {}, qo = {};
    KvRope r = {};
    int rc;
    if ((rc = check_cache(cache, &c)) || (rc = check_batch(batch, c.shift, &b)))
        return rc;
    if (batch->tokens == 0)
        return MXFP4_OK;
    if ((rc = check_tensor(k, "k", &kt)) || (rc = check_tensor(v, "v", &vt)))
        return rc;
    if (q) {
        if ((rc = check_tensor(q, "q", &qt)) || (rc = check_tensor(q_out, "q_out", &qo)))
            return rc;
        if (q_heads < 1 || q_heads > 65535)
            return fail(MXFP4_ERR_SHAPE, "q_heads=%lld out of range [1, 65535]", (long long)q_heads);
        if (qt.p == qo.p)
            return fail(MXFP4_ERR_ARG, "q_out must not be q (a pair's halves are turned by different threads)");
    } else {
        q_heads = 0;
    }
    if (rope && rope->dim) {
        if (!rope->cos_f32 || !rope->sin_f32)
            return fail(MXFP4_ERR_NULL, "cos_f32 or sin_f32 is NULL");
        if (rope->dim < 16 || rope->dim % 16 || rope->dim > cache->dim)
            return fail(MXFP4_ERR_SHAPE, "rotary dim=%lld must be a multiple of 16 up to the head dimension %d", (long long)rope->dim, cache->dim);
        if (rope->length < 1 || rope->length > 0x7FFFFFFF)
            return fail(MXFP4_ERR_SHAPE, "rotary length=%lld out of range", (long long)rope->length);
        if (!aligned(rope->cos_f32, 16) || !aligned(rope->sin_f32, 16) || !aligned(rope->positions, 4))
            return fail(MXFP4_ERR_ALIGN, "cos_f32 and sin_f32 must be 16-byte aligned, positions 4-byte");
        r = {rope->cos_f32, rope->sin_f32, rope->positions, (int)rope->length, (int)rope->dim};
    }
    return launched(launch_kv_append(c, b, kt, vt, qt, qo, (int)q_heads, r, static_cast<hipStream_t>(stream)), "cache append launch");
}

int mxfp4_kv_read(const mxfp4_kv_cache* cache, const mxfp4_kv_rows* batch, const mxfp4_kv_tensor* k_out,
                  const mxfp4_kv_tensor* v_out, void* stream)
{
    begin_call();
    KvView c;
    KvBatch b = {};
    KvTensor kt = {}, vt = {};
    int rc;
    if ((rc = check_cache(cache, &c)) || (rc = check_batch(batch, c.shift, &b)))
        return rc;
    if (batch->tokens == 0)
        return MXFP4_OK;
    if (!k_out && !v_out)
        return fail(MXFP4_ERR_NULL, "k_out and v_out are both NULL");
    if ((k_out && (rc = check_tensor(k_out, "k_out", &kt))) || (v_out && (rc = check_tensor(v_out, "v_out", &vt))))
        return rc;
    return launched(launch_kv_read(c, b, kt, vt, static_cast<hipStream_t>(stream)), "cache read launch");
}

size_t mxfp4_kv_attention_workspace_bytes(const mxfp4_kv_cache* cache, const mxfp4_kv_rows* batch, int64_t q_heads)
{
    KvView c;
    DeviceInfo dev;
    if (check_cache(cache, &c) || !batch || batch->tokens < 0 || batch->rows < 0 || q_heads < 1 || q_heads > 65535 || q_heads % c.heads)
        return 0;
    if (device_info(&dev) != MXFP4_OK) {
        dev.cus = 256;
        dev.lds_bytes = 160 * 1024;
        begin_call();
    }
    return MXFP4_KV_COUNTERS * sizeof(uint32_t) +
           kv_attend_part_bytes(c.nb, (int)(q_heads / c.heads), batch->tokens, batch->rows, dev);
}

int mxfp4_kv_attention(const mxfp4_kv_cache* cache, const mxfp4_kv_rows* batch, const mxfp4_kv_attention_args* args,
                       void* workspace, size_t workspace_bytes, void* stream)
{
    begin_call();
    KvAttend a = {};
    int rc;
    if ((rc = check_cache(cache, &a.c)) || (rc = check_batch(batch, a.c.shift, &a.b)))
        return rc;
    if (!args)
        return fail(MXFP4_ERR_NULL, "args is NULL");
    if (batch->tokens == 0)
        return MXFP4_OK;
    if ((rc = check_tensor(&args->q, "q", &a.q)) || (rc = check_tensor(&args->out, "out", &a.out)))
        return rc;
    if (args->q_heads < 1 || args->q_heads > 65535 || args->q_heads % cache->heads)
        return fail(MXFP4_ERR_SHAPE, "q_heads=%lld must be a multiple of the cache's %d heads", (long long)args->q_heads, cache->heads);
    if (args->q_heads / cache->heads * batch->tokens > 0x3FFFFFFF)
        return fail(MXFP4_ERR_SHAPE, "%lld tokens of %lld query heads are too many", (long long)batch->tokens, (long long)args->q_heads);
    if (args->window < 0 || args->window > 0x7FFFFFFF)
        return fail(MXFP4_ERR_SHAPE, "window=%lld out of range", (long long)args->window);
    if (!(args->scale > 0.f) || !isfinite(args->scale))
        return fail(MXFP4_ERR_ARG, "scale must be a positive number");
    if (!aligned(args->lse_f32, 4) || !aligned(args->tree, 8))
        return fail(MXFP4_ERR_ALIGN, "lse_f32 must be 4-byte aligned, tree 8-byte");
    DeviceInfo dev;
    if ((rc = device_info(&dev)))
        return rc;
    const size_t need = mxfp4_kv_attention_workspace_bytes(cache, batch, args->q_heads);
    if (!workspace || workspace_bytes < need)
        return fail(MXFP4_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, workspace ? workspace_bytes : (size_t)0);
    if (!aligned(workspace, 16))
        return fail(MXFP4_ERR_ALIGN, "workspace must be 16-byte aligned");
    a.lse = args->lse_f32;
    a.tree = args->tree;
    a.group = (int)(args->q_heads / cache->heads);
    a.causal = args->causal != 0;
    // Positions lie in [-2^30, 2^30): a wider window hides nothing, and their differences stay within 32 bits.
    a.window = (int)(args->window < (1 << 30) ? args->window : 1 << 30);
    a.scale = args->scale * 1.4426950408889634f;
    a.counters = static_cast<uint32_t*>(workspace);
    a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + MXFP4_KV_COUNTERS * sizeof(uint32_t));
    return launched(launch_kv_attend(a, dev, static_cast<hipStream_t>(stream)), "cache attention launch");
}

int mxfp4_kv_fork(const mxfp4_kv_pool* pool, const int32_t* src, const int32_t* dst, int64_t count, void* stream)
{
    begin_call();
    KvPool p;
    const int rc = check_pool(pool, count, &p);
    if (rc || count == 0)
        return rc;
    if (!src || !dst)
        return fail(MXFP4_ERR_NULL, "src or dst is NULL");
    if (!aligned(src, 4) || !aligned(dst, 4))
        return fail(MXFP4_ERR_ALIGN, "src and dst must be 4-byte aligned");
    return launched(launch_kv_fork(p, src, dst, (int)count, static_cast<hipStream_t>(stream)), "fork launch");
}

int mxfp4_kv_extend(const mxfp4_kv_pool* pool, const mxfp4_kv_cache* cache, const int32_t* rows_list, const int32_t* add,
                    int64_t count, int32_t* copies, int32_t* missing, void* stream)
{
    begin_call();
    KvPool p;
    KvView c = {};
    int rc = check_pool(pool, count, &p);
    if (rc)
        return rc;
    if (count > kKvMaxRows)
        return fail(MXFP4_ERR_SHAPE, "count=%lld: at most %d rows in one call", (long long)count, kKvMaxRows);
    if (cache) {
        if ((rc = check_cache(cache, &c)))
            return rc;
        if (cache->pages != pool->pages || cache->page != pool->page)
            return fail(MXFP4_ERR_SHAPE, "the cache has %lld pages of %d tokens, the pool %lld of %lld", (long long)cache->pages, cache->page,
                        (long long)pool->pages, (long long)pool->page);
    }
    if (!copies || !missing || (count && (!rows_list || !add)))
        return fail(MXFP4_ERR_NULL, "rows_list, add, copies or missing is NULL");
    if (!aligned(rows_list, 4) || !aligned(add, 4) || !aligned(copies, 4) || !aligned(missing, 4))
        return fail(MXFP4_ERR_ALIGN, "rows_list, add, copies and missing must be 4-byte aligned");
    hipStream_t s = static_cast<hipStream_t>(stream);
    rc = launched(launch_kv_extend(p, rows_list, add, (int)count, copies, missing, s), "extend launch");
    if (rc || !cache || count == 0)
        return rc;
    return launched(launch_kv_copy(c, copies, copies + 1, 2, (int)count, rows_list, p.rows, p.lens, add, s), "page copy launch");
}

int mxfp4_kv_release(const mxfp4_kv_pool* pool, const int32_t* rows_list, const int32_t* keep, int64_t count, void* stream)
{
    begin_call();
    KvPool p;
    const int rc = check_pool(pool, count, &p);
    if (rc || count == 0)
        return rc;
    if (!rows_list || !keep)
        return fail(MXFP4_ERR_NULL, "rows_list or keep is NULL");
    if (!aligned(rows_list, 4) || !aligned(keep, 4))
        return fail(MXFP4_ERR_ALIGN, "rows_list and keep must be 4-byte aligned");
    return launched(launch_kv_release(p, rows_list, keep, (int)count, static_cast<hipStream_t>(stream)), "release launch");
}

int mxfp4_kv_compact(const mxfp4_kv_cache* cache, const int32_t* table, int64_t ldt, int64_t width, const int32_t* base,
                     const int32_t* keep, int64_t ldk, const int32_t* counts, int64_t rows, void* stream)
{
    begin_call();
    KvView c;
    int rc = check_cache(cache, &c);
    if (rc)
        return rc;
    if (rows < 0 || rows > (1 << 20) || ldk < 0 || ldk > 0x3FFFFFFF)
        return fail(MXFP4_ERR_SHAPE, "rows=%lld or ldk=%lld out of range", (long long)rows, (long long)ldk);
    if (rows == 0 || ldk == 0)
        return MXFP4_OK;
    if ((rc = check_table(table, ldt, width, c.shift)))
        return rc;
    if (!base || !keep || !counts)
        return fail(MXFP4_ERR_NULL, "base, keep or counts is NULL");
    if (!aligned(base, 4) || !aligned(keep, 4) || !aligned(counts, 4))
        return fail(MXFP4_ERR_ALIGN, "base, keep and counts must be 4-byte aligned");
    return launched(launch_kv_compact(c, table, ldt, (int)width, base, keep, (int)ldk, counts, (int)rows, static_cast<hipStream_t>(stream)),
                    "compact launch");
}

int mxfp4_kv_copy_pages(const mxfp4_kv_cache* cache, const int32_t* src, const int32_t* dst, int64_t count, void* stream)
{
    begin_call();
    KvView c;
    const int rc = check_cache(cache, &c);
    if (rc)
        return rc;
    if (count < 0 || count > 0x7FFFFFFF)
        return fail(MXFP4_ERR_SHAPE, "count=%lld out of range", (long long)count);
    if (count == 0)
        return MXFP4_OK;
    if (!src || !dst)
        return fail(MXFP4_ERR_NULL, "src or dst is NULL");
    if (!aligned(src, 4) || !aligned(dst, 4))
        return fail(MXFP4_ERR_ALIGN, "src and dst must be 4-byte aligned");
    return launched(launch_kv_copy(c, src, dst, 1, (int)count, nullptr, 0, nullptr, nullptr, static_cast<hipStream_t>(stream)),
                    "page copy launch");
}

}  // extern "C"
