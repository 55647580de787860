// The way from a Python call of the paged cache to its launch, for the call as programs make it; as in host.cpp, anything else returns
// None, and the binding's own checks and messages take the call.
//
// What bounds it: a step's calls run 3 to 10 us on the device, and building their five structures through ctypes took longer.
#include "host.h"

namespace mxfp4_host {

namespace {

struct Call {
    c10::Device device = c10::Device(c10::kCUDA, 0);
    void* stream = nullptr;
    mxfp4_kv_cache cache{};
    mxfp4_kv_rows rows{};
};

bool modes() { return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set(); }

// The cache: a tuple of four uint8 tensors, each contiguous within a page.
bool cache_of(PyObject* o, Call* c)
{
    if (modes() || !PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4)
        return false;
    PyObject* first = PyTuple_GET_ITEM(o, 0);
    if (!THPVariable_CheckExact(first) || !THPVariable_Unpack(first).is_cuda())
        return false;
    const c10::DeviceIndex at = c10::hip::current_device();
    c->device = c10::Device(c10::kCUDA, at);
    c->stream = c10::hip::getCurrentHIPStream(at).stream();
    const at::Tensor* x[4];
    for (int i = 0; i < 4; ++i) {
        x[i] = plain(PyTuple_GET_ITEM(o, i), at::kByte, c->device);
        if (!x[i] || x[i]->dim() != 4)
            return false;
    }
    const int64_t pages = x[0]->size(0), heads = x[0]->size(1), page = x[0]->size(2), half = x[0]->size(3);
    if (half < 16 || half % 16 || half > 4096 || heads < 1 || heads > 65535 || page < 1 || page > 1024)
        return false;
    for (int i = 0; i < 4; ++i) {
        const int64_t wide = i % 2 ? half / 16 : half;
        if (x[i]->size(0) != pages || x[i]->size(1) != heads || x[i]->size(2) != page || x[i]->size(3) != wide || x[i]->stride(1) != page * wide ||
            x[i]->stride(2) != wide || x[i]->stride(3) != 1 || x[i]->stride(0) != x[i % 2]->stride(0))
            return false;
    }
    c->cache = {x[0]->data_ptr(), x[1]->data_ptr(), x[2]->data_ptr(), x[3]->data_ptr(), pages,
                pages > 1 ? x[0]->stride(0) : heads * page * half, pages > 1 ? x[1]->stride(0) : heads * page * (half / 16),
                (int32_t)heads, (int32_t)page, (int32_t)(half * 2), 0};
    return true;
}

// int32 [n]; n < 0: any.
const at::Tensor* ints(PyObject* o, c10::Device device, int64_t n)
{
    const at::Tensor* t = plain(o, at::kInt, device);
    return t && t->dim() == 1 && t->is_contiguous() && (n < 0 || t->size(0) == n) ? t : nullptr;
}

const at::Tensor* table_of(PyObject* o, c10::Device device, int64_t* ldt)
{
    const at::Tensor* t = plain(o, at::kInt, device);
    if (!t || t->dim() != 2 || (t->size(1) > 1 && t->stride(1) != 1))
        return nullptr;
    *ldt = t->size(0) > 1 ? t->stride(0) : t->size(1);
    return t;
}

bool rows_of(PyObject* table, PyObject* lens, PyObject* starts, int64_t tokens, Call* c)
{
    int64_t ldt;
    const at::Tensor* t = table_of(table, c->device, &ldt);
    if (!t)
        return false;
    const int64_t rows = t->size(0);
    const at::Tensor *n = ints(lens, c->device, rows), *s = starts == Py_None ? nullptr : ints(starts, c->device, rows + 1);
    if (!n || (starts != Py_None && !s))
        return false;
    c->rows = {(const int32_t*)t->data_ptr(), ldt, t->size(1), (const int32_t*)n->data_ptr(), s ? (const int32_t*)s->data_ptr() : nullptr,
               rows, tokens};
    return true;
}

// BF16 [tokens, heads, dim]; tokens, heads < 0: any.
const at::Tensor* heads_of(PyObject* o, c10::Device device, int64_t tokens, int64_t heads, int64_t dim, mxfp4_kv_tensor* d)
{
    const at::Tensor* t = plain(o, at::kBFloat16, device);
    if (!t || t->dim() != 3 || (tokens >= 0 && t->size(0) != tokens) || (heads >= 0 && t->size(1) != heads) || t->size(2) != dim || t->stride(2) != 1)
        return nullptr;
    *d = {t->data_ptr(), t->size(0) > 1 ? t->stride(0) : 0, t->size(1) > 1 ? t->stride(1) : 0};
    return t;
}

mxfp4_kv_tensor whole(const at::Tensor& t) { return {t.data_ptr(), t.size(1) * t.size(2), t.size(2)}; }

PyObject* wrap_true(const at::Tensor*) { Py_RETURN_TRUE; }

bool counted(Py_ssize_t count, Py_ssize_t want, const char* what)
{
    if (count != want)
        PyErr_Format(PyExc_TypeError, "%s: %zd arguments", what, want);
    return count == want;
}

// kv_append(cache, k, v, table, lens, starts, q, rope, positions) -> the turned queries, True without any, or None
PyObject* kv_append(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    if (!counted(count, 9, "kv_append"))
        return nullptr;
    Call c;
    mxfp4_kv_tensor k, v, q;
    if (!cache_of(args[0], &c))
        return left();
    const int64_t dim = c.cache.dim;
    const at::Tensor* kt = heads_of(args[1], c.device, -1, c.cache.heads, dim, &k);
    if (!kt || !heads_of(args[2], c.device, kt->size(0), c.cache.heads, dim, &v) || !rows_of(args[3], args[4], args[5], kt->size(0), &c))
        return left();
    const at::Tensor* qt = nullptr;
    if (args[6] != Py_None && !(qt = heads_of(args[6], c.device, kt->size(0), -1, dim, &q)))
        return left();
    mxfp4_kv_rope rope{};
    if (args[7] != Py_None) {
        if (!PyTuple_CheckExact(args[7]) || PyTuple_GET_SIZE(args[7]) != 2)
            return left();
        const at::Tensor *cos = plain(PyTuple_GET_ITEM(args[7], 0), at::kFloat, c.device), *sin = plain(PyTuple_GET_ITEM(args[7], 1), at::kFloat, c.device);
        if (!cos || !sin || cos->dim() != 2 || cos->sizes() != sin->sizes() || !cos->is_contiguous() || !sin->is_contiguous())
            return left();
        rope = {(const float*)cos->data_ptr(), (const float*)sin->data_ptr(), nullptr, cos->size(0), 2 * cos->size(1)};
        if (args[8] != Py_None) {
            const at::Tensor* p = ints(args[8], c.device, kt->size(0));
            if (!p)
                return left();
            rope.positions = (const int32_t*)p->data_ptr();
        }
    } else if (args[8] != Py_None) {
        return left();
    }
    at::Tensor out;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        mxfp4_kv_tensor to{};
        if (qt) {
            out = fresh({qt->size(0), qt->size(1), dim}, at::kBFloat16, c.device);
            to = whole(out);
        }
        rc = mxfp4_kv_append(&c.cache, &c.rows, &k, &v, qt ? &q : nullptr, qt ? &to : nullptr, qt ? qt->size(1) : 0,
                             args[7] != Py_None ? &rope : nullptr, c.stream);
    }
    return finish(rc, qt ? wrap_one : wrap_true, &out);
    END_HANDLE_TH_ERRORS
}

// kv_read(cache, table, lens, tokens, starts) -> (k, v), or None
PyObject* kv_read(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    if (!counted(count, 5, "kv_read"))
        return nullptr;
    Call c;
    int tokens;
    if (!small(args[3], &tokens) || tokens < 0 || !cache_of(args[0], &c) || !rows_of(args[1], args[2], args[4], tokens, &c))
        return left();
    at::Tensor out[2];
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        for (auto& t : out)
            t = fresh({tokens, c.cache.heads, c.cache.dim}, at::kBFloat16, c.device);
        const mxfp4_kv_tensor k = whole(out[0]), v = whole(out[1]);
        rc = mxfp4_kv_read(&c.cache, &c.rows, &k, &v, c.stream);
    }
    return finish(rc, wrap_two, out);
    END_HANDLE_TH_ERRORS
}

// kv_attention(q, cache, table, lens, starts, scale, causal, window, tree, lse, workspaces) -> out or (out, lse), or None.  workspaces: the
// binding's, by stream and device; a stream that has none yet, or too small a one, and a captured call are left to the binding.
PyObject* kv_attention(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    if (!counted(count, 11, "kv_attention"))
        return nullptr;
    Call c;
    mxfp4_kv_attention_args a{};
    int window;
    if (!small(args[7], &window) || !PyDict_Check(args[10]) || !cache_of(args[1], &c))
        return left();
    const at::Tensor* q = heads_of(args[0], c.device, -1, -1, c.cache.dim, &a.q);
    if (!q || !rows_of(args[2], args[3], args[4], q->size(0), &c))
        return left();
    if (args[8] != Py_None) {
        const at::Tensor* tree = plain(args[8], at::kLong, c.device);
        if (!tree || tree->dim() != 1 || tree->size(0) != q->size(0) || !tree->is_contiguous())
            return left();
        a.tree = (const uint64_t*)tree->data_ptr();
    }
    if (args[5] == Py_None) {
        a.scale = (float)(1.0 / sqrt((double)c.cache.dim));
    } else {
        const double s = PyFloat_Check(args[5]) ? PyFloat_AS_DOUBLE(args[5]) : 0.0;
        if (!(s > 0.0))
            return left();
        a.scale = (float)s;
    }
    if ((args[6] != Py_True && args[6] != Py_False) || (args[9] != Py_True && args[9] != Py_False))
        return left();                                  // (any other truth value is the binding's to read)
    a.causal = args[6] == Py_True;
    a.window = window;
    a.q_heads = q->size(1);
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing((hipStream_t)c.stream, &capture) != hipSuccess || capture != hipStreamCaptureStatusNone)
        return left();
    PyObject* key = PyLong_FromLongLong((long long)((uintptr_t)c.stream * 64 + (uintptr_t)c.device.index()));
    PyObject* held = key ? PyDict_GetItemWithError(args[10], key) : nullptr;
    Py_XDECREF(key);
    const at::Tensor* ws = held ? plain(held, at::kByte, c.device) : nullptr;
    const size_t need = mxfp4_kv_attention_workspace_bytes(&c.cache, &c.rows, a.q_heads);
    if (!ws || need == 0 || (size_t)ws->numel() < need)
        return left();
    const at::Tensor space = *ws;                       // (kept while the lock is released)
    const bool lse = args[9] == Py_True;
    at::Tensor out[2];
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        out[0] = fresh({q->size(0), q->size(1), q->size(2)}, at::kBFloat16, c.device);
        a.out = whole(out[0]);
        if (lse) {
            out[1] = fresh({q->size(0), q->size(1)}, at::kFloat, c.device);
            a.lse_f32 = (float*)out[1].data_ptr();
        }
        rc = mxfp4_kv_attention(&c.cache, &c.rows, &a, space.data_ptr(), (size_t)space.numel(), c.stream);
    }
    return finish(rc, lse ? wrap_two : wrap_one, out);
    END_HANDLE_TH_ERRORS
}

// kv_pages(what, refs, free, cache, table, lens, rows, numbers) -> True (what 0: fork, 1: release) or what is missing (2: extend), or None
PyObject* kv_pages(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    if (!counted(count, 8, "kv_pages"))
        return nullptr;
    Call c;
    int what;
    int64_t ldt;
    if (!small(args[0], &what) || !cache_of(args[3], &c))
        return left();
    const at::Tensor *refs = ints(args[1], c.device, -1), *table = table_of(args[4], c.device, &ldt);
    if (!refs || !table)
        return left();
    const int64_t pages = refs->size(0);
    const at::Tensor *bits = ints(args[2], c.device, (pages + 31) / 32), *lens = ints(args[5], c.device, table->size(0)),
                     *a = ints(args[6], c.device, -1), *b = a ? ints(args[7], c.device, a->size(0)) : nullptr;
    if (!bits || !lens || !a || !b)
        return left();
    const mxfp4_kv_pool pool = {(int32_t*)refs->data_ptr(), (uint32_t*)bits->data_ptr(), pages, c.cache.page, (int32_t*)table->data_ptr(), ldt,
                                table->size(1), table->size(0), (int32_t*)lens->data_ptr()};
    const int64_t n = a->size(0);
    const int32_t *first = (const int32_t*)a->data_ptr(), *second = (const int32_t*)b->data_ptr();
    at::Tensor missing, copies;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        if (what == 2) {
            missing = fresh({1}, at::kInt, c.device);
            copies = fresh({2 * n + 1}, at::kInt, c.device);
            rc = mxfp4_kv_extend(&pool, &c.cache, first, second, n, (int32_t*)copies.data_ptr(), (int32_t*)missing.data_ptr(), c.stream);
        } else {
            rc = (what == 0 ? mxfp4_kv_fork : mxfp4_kv_release)(&pool, first, second, n, c.stream);
        }
    }
    return finish(rc, what == 2 ? wrap_one : wrap_true, &missing);
    END_HANDLE_TH_ERRORS
}

// kv_compact(cache, table, base, keep, counts) -> True, or None
PyObject* kv_compact(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    if (!counted(count, 5, "kv_compact"))
        return nullptr;
    Call c;
    int64_t ldt;
    const at::Tensor* table = cache_of(args[0], &c) ? table_of(args[1], c.device, &ldt) : nullptr;
    if (!table)
        return left();
    const int64_t rows = table->size(0);
    const at::Tensor *base = ints(args[2], c.device, rows), *keep = plain(args[3], at::kInt, c.device), *counts = ints(args[4], c.device, rows);
    if (!base || !counts || !keep || keep->dim() != 2 || keep->size(0) != rows || !keep->is_contiguous())
        return left();
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        rc = mxfp4_kv_compact(&c.cache, (const int32_t*)table->data_ptr(), ldt, table->size(1), (const int32_t*)base->data_ptr(),
                              (const int32_t*)keep->data_ptr(), keep->size(1), (const int32_t*)counts->data_ptr(), rows, c.stream);
    }
    return finish(rc, wrap_true, nullptr);
    END_HANDLE_TH_ERRORS
}

}  // namespace

PyMethodDef kv_methods[] = {
    {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, nullptr},
    {"kv_read", (PyCFunction)(void (*)(void))kv_read, METH_FASTCALL, nullptr},
    {"kv_attention", (PyCFunction)(void (*)(void))kv_attention, METH_FASTCALL, nullptr},
    {"kv_pages", (PyCFunction)(void (*)(void))kv_pages, METH_FASTCALL, nullptr},
    {"kv_compact", (PyCFunction)(void (*)(void))kv_compact, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

}  // namespace mxfp4_host
