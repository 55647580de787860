// The way from a Python call of what surrounds a layer's products to its launch, for the call as programs make it; as in host.cpp,
// anything else returns None, and the binding's own checks and messages take the call.
#include "host.h"

namespace mxfp4_host {

namespace {

struct Where {
    c10::Device device = c10::Device(c10::kCUDA, 0);
    void* stream = nullptr;
};

// Where a call runs: the current device, which its first tensor has to be on.
bool where(PyObject* first, Where* w)
{
    if (at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set() || !THPVariable_CheckExact(first) ||
        !THPVariable_Unpack(first).is_cuda())
        return false;
    const c10::DeviceIndex at = c10::hip::current_device();
    w->device = c10::Device(c10::kCUDA, at);
    w->stream = c10::hip::getCurrentHIPStream(at).stream();
    return true;
}

struct Rows {
    void* at = nullptr;
    int64_t ld = 0;
};

// BF16 [m, k], columns side by side; m, k < 0: any.
const at::Tensor* rows_of(PyObject* o, c10::Device device, int64_t m, int64_t k, Rows* r)
{
    const at::Tensor* t = plain(o, at::kBFloat16, device);
    if (!t || t->dim() != 2 || (m >= 0 && t->size(0) != m) || (k >= 0 && t->size(1) != k) || (t->size(1) > 1 && t->stride(1) != 1))
        return nullptr;
    *r = {t->data_ptr(), t->size(0) > 1 ? t->stride(0) : t->size(1)};
    return t;
}

// The same, or nothing where None is given.
bool maybe_rows(PyObject* o, c10::Device device, int64_t m, int64_t k, Rows* r) { return o == Py_None || rows_of(o, device, m, k, r); }

// A contiguous tensor of these sizes (b < 0: one dimension).
const at::Tensor* whole_of(PyObject* o, at::ScalarType type, c10::Device device, int64_t a, int64_t b = -1)
{
    const at::Tensor* t = plain(o, type, device);
    return t && t->dim() == (b < 0 ? 1 : 2) && t->size(0) == a && (b < 0 || t->size(1) == b) && t->is_contiguous() ? t : nullptr;
}

bool counted(Py_ssize_t count, Py_ssize_t want, const char* what)
{
    if (count != want)
        PyErr_Format(PyExc_TypeError, "%s: %zd arguments", what, want);
    return count == want;
}

// y, sum, codes and scales of a norm, None for what was not made.
PyObject* wrap_norm(const at::Tensor* t)
{
    PyObject* tuple = PyTuple_New(4);
    for (int i = 0; tuple && i < 4; ++i) {
        PyObject* item = t[i].defined() ? THPVariable_Wrap(t[i]) : Py_NewRef(Py_None);
        if (!item) {
            Py_DECREF(tuple);
            return nullptr;
        }
        PyTuple_SET_ITEM(tuple, i, item);
    }
    return tuple;
}

// rms_norm(x, weight, residual, eps, bf16, e4m3) -> (y, sum, q8, s), or None
PyObject* rms_norm(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    if (!counted(count, 6, "rms_norm"))
        return nullptr;
    Where w;
    Rows x, r;
    if (!where(args[0], &w) || !PyFloat_Check(args[3]))
        return left();
    const at::Tensor* t = rows_of(args[0], w.device, -1, -1, &x);
    if (!t)
        return left();
    const int64_t m = t->size(0), k = t->size(1);
    const bool bf16 = args[4] == Py_True, e4m3 = args[5] == Py_True;
    if (m < 1 || k < 8 || !maybe_rows(args[2], w.device, m, k, &r))
        return left();
    const void* weight = nullptr;
    if (args[1] != Py_None) {
        const at::Tensor* g = whole_of(args[1], at::kBFloat16, w.device, k);
        if (!g)
            return left();
        weight = g->data_ptr();
    }
    const float eps = (float)PyFloat_AS_DOUBLE(args[3]);
    at::Tensor out[4];
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        if (bf16)
            out[0] = fresh({m, k}, at::kBFloat16, w.device);
        if (r.at)
            out[1] = fresh({m, k}, at::kBFloat16, w.device);
        if (e4m3) {
            out[2] = fresh({m, k}, at::kByte, w.device);
            out[3] = fresh({m, k / 32}, at::kByte, w.device);
        }
        auto at = [](const at::Tensor& v) { return v.defined() ? v.data_ptr() : nullptr; };
        rc = mxfp4_rms_norm(x.at, m, k, x.ld, r.at, r.ld, weight, eps, at(out[1]), k, at(out[0]), k, at(out[2]), at(out[3]), w.stream);
    }
    return finish(rc, wrap_norm, out);
    END_HANDLE_TH_ERRORS
}

// e4m3_dequant(q8, s) -> w, or None
PyObject* e4m3_dequant(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    if (!counted(count, 2, "e4m3_dequant"))
        return nullptr;
    Where w;
    if (!where(args[0], &w))
        return left();
    const at::Tensor* q = plain(args[0], at::kByte, w.device);
    if (!q || q->dim() != 2 || !q->is_contiguous())
        return left();
    const int64_t m = q->size(0), k = q->size(1);
    const at::Tensor* s = m < 1 || k < 32 || k % 32 ? nullptr : whole_of(args[1], at::kByte, w.device, m, k / 32);
    if (!s)
        return left();
    at::Tensor y;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        y = fresh({m, k}, at::kBFloat16, w.device);
        rc = mxfp4_e4m3_dequant(q->data_ptr(), s->data_ptr(), m, k, y.data_ptr(), k, w.stream);
    }
    return finish(rc, wrap_one, &y);
    END_HANDLE_TH_ERRORS
}

// w4a8(x8, xs, q, s, bias, act, residual) -> y, or None
PyObject* w4a8(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    if (!counted(count, 7, "w4a8"))
        return nullptr;
    Where w;
    Rows r;
    int act;
    if (!small(args[5], &act) || !where(args[0], &w))
        return left();
    const at::Tensor *x = plain(args[0], at::kByte, w.device), *q = plain(args[2], at::kByte, w.device);
    if (!x || !q || x->dim() != 2 || q->dim() != 2 || !x->is_contiguous() || !q->is_contiguous())
        return left();
    const int64_t m = x->size(0), k = x->size(1), n = q->size(0), c = act == MXFP4_ACT_SWIGLU ? n / 2 : n;
    if (m < 1 || n < 1 || k < 32 || k % 32 || q->size(1) != k / 2)
        return left();
    const at::Tensor *xs = whole_of(args[1], at::kByte, w.device, m, k / 32), *s = whole_of(args[3], at::kByte, w.device, n, k / 32);
    if (!xs || !s || !maybe_rows(args[6], w.device, m, c, &r))
        return left();
    const void* bias = nullptr;
    if (args[4] != Py_None) {
        const at::Tensor* b = whole_of(args[4], at::kBFloat16, w.device, n);
        if (!b)
            return left();
        bias = b->data_ptr();
    }
    at::Tensor y;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        y = fresh({m, c}, at::kBFloat16, w.device);
        rc = mxfp4_w4a8_gemm(x->data_ptr(), xs->data_ptr(), m, q->data_ptr(), s->data_ptr(), n, k, bias, act, r.at, r.ld, y.data_ptr(), c,
                             w.stream);
    }
    return finish(rc, wrap_one, &y);
    END_HANDLE_TH_ERRORS
}

// lora(x, a, b, ids, base, scales) -> y, or None
PyObject* lora(PyObject*, PyObject* const* args, Py_ssize_t count)
{
    HANDLE_TH_ERRORS
    if (!counted(count, 6, "lora"))
        return nullptr;
    Where w;
    Rows x, base;
    if (!where(args[0], &w))
        return left();
    const at::Tensor *t = rows_of(args[0], w.device, -1, -1, &x), *a = plain(args[1], at::kBFloat16, w.device),
                     *b = plain(args[2], at::kBFloat16, w.device);
    if (!t || !a || !b || a->dim() != 3 || b->dim() != 3 || !a->is_contiguous() || !b->is_contiguous())
        return left();
    const int64_t m = t->size(0), k = t->size(1), many = a->size(0), rank = a->size(1), n = b->size(1);
    if (m < 1 || a->size(2) != k || b->size(0) != many || b->size(2) != rank)
        return left();
    const at::Tensor* ids = whole_of(args[3], at::kInt, w.device, m);
    if (!ids || !maybe_rows(args[4], w.device, m, n, &base))
        return left();
    const float* scales = nullptr;
    if (args[5] != Py_None) {
        const at::Tensor* f = whole_of(args[5], at::kFloat, w.device, many);
        if (!f)
            return left();
        scales = (const float*)f->data_ptr();
    }
    const size_t need = mxfp4_lora_workspace_bytes(m, k, rank);
    if (need == 0)
        return left();
    at::Tensor y, ws;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        y = fresh({m, n}, at::kBFloat16, w.device);
        ws = fresh({(int64_t)need}, at::kByte, w.device);
        rc = mxfp4_lora(t->data_ptr(), m, x.ld, a->data_ptr(), b->data_ptr(), many, rank, n, k, (const int32_t*)ids->data_ptr(), scales,
                        base.at, base.ld, y.data_ptr(), n, ws.data_ptr(), need, w.stream);
    }
    return finish(rc, wrap_one, &y);
    END_HANDLE_TH_ERRORS
}

}  // namespace

PyMethodDef layer_methods[] = {
    {"rms_norm", (PyCFunction)(void (*)(void))rms_norm, METH_FASTCALL, nullptr},
    {"w4a8", (PyCFunction)(void (*)(void))w4a8, METH_FASTCALL, nullptr},
    {"lora", (PyCFunction)(void (*)(void))lora, METH_FASTCALL, nullptr},
    {"e4m3_dequant", (PyCFunction)(void (*)(void))e4m3_dequant, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

}  // namespace mxfp4_host
